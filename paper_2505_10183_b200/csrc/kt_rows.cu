// kt_rows.cu -- operators on rows of activations that a data-parallel worker runs to obtain the
// gradients the library synchronises: layer norm forward and backward (with the reduction of the
// weight's and the bias' gradient over all rows), GELU / SiLU forward and backward, and the 8-bit
// checkpoints that both can leave for the backward pass.  Contracts: include/kaitian.h.
//
// All of it is bound by memory: a row is read once with 128-bit loads, stays in registers as fp32
// for its statistics and its result, and is written once.  Rows whose address or width does not
// allow 128-bit accesses take the same kernels with element accesses (template argument WIDE).
//
// 8-bit checkpoints.  A block of KT_CKPT_BLOCK = 128 columns of a row shares one fp32 scale:
//   top = max |x|,  scale = top / 127,  code = rint(x * 127 / top) in -127 ... 127,
// so that a value is off by at most scale / 2.  A block with top < 2^-100 is kept as zeros (127 / top
// must not overflow); one with an infinity or a NaN gets scale NaN, so that it restores as NaN
// and is not silently cut off.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <climits>
#include <cmath>

#include "kt_internal.h"

using namespace ktd;

namespace {

constexpr int BLOCK = KT_CKPT_BLOCK;
constexpr int E = 16;                    // row elements that a thread keeps in registers
constexpr int GROUP_MAX = 512;           // threads on one row at most
constexpr int64_t ROW_MAX = E * GROUP_MAX;   // wider rows are read again instead of kept
constexpr int PARTS_MAX = 592;           // rows of partial weight gradients: four to an SM
constexpr float SMALLEST = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// V consecutive elements of a row in one 16-byte vector, or what there is of them.
template <typename T>
struct Elems;
template <>
struct Elems<float> {
    static constexpr int V = 4;
    __device__ static void widen(const uint4 &r, float (&x)[4]) {
        x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
    }
    __device__ static uint4 narrow(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static float one(float x) { return x; }
    __device__ static float up(float x) { return x; }
};
template <>
struct Elems<__nv_bfloat16> {
    static constexpr int V = 8;
    __device__ static void widen(const uint4 &r, float (&x)[8]) {
        const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    __device__ static uint4 narrow(const float (&x)[8]) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned *>(&p);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __nv_bfloat16 one(float x) { return __float2bfloat16_rn(x); }
    __device__ static float up(__nv_bfloat16 x) { return __bfloat162float(x); }
};

template <typename T, bool WIDE>
__device__ __forceinline__ void load_row(const T *row, int64_t col, int64_t cols, float (&x)[Elems<T>::V]) {
    constexpr int V = Elems<T>::V;
    if constexpr (WIDE) {
        if (col < cols) {
            Elems<T>::widen(load16(row + col), x);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = col + i < cols ? Elems<T>::up(row[col + i]) : 0.0f;
    }
}

template <typename T, bool WIDE>
__device__ __forceinline__ void store_row(T *row, int64_t col, int64_t cols, const float (&x)[Elems<T>::V]) {
    constexpr int V = Elems<T>::V;
    if constexpr (WIDE) {
        if (col < cols) *reinterpret_cast<uint4 *>(row + col) = Elems<T>::narrow(x);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col + i < cols) row[col + i] = Elems<T>::one(x[i]);
    }
}

// V columns of a weight or bias (fp32 or bf16, any alignment); `missing` where there is none.
template <int V>
__device__ __forceinline__ void load_param(const void *p, bool bf16, int64_t col, int64_t cols, float missing, float (&w)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = missing;
        if (p != nullptr && col + i < cols)
            w[i] = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[col + i]) : static_cast<const float *>(p)[col + i];
    }
}

// The V codes of one vector and the scale of its block.  The 128 / V lanes that hold a block are
// neighbours; all lanes of the warp call it.  Columns at or past `cols` hold zeros.
template <int V>
__device__ __forceinline__ void encode(const float (&x)[V], uint2 *codes, float *scale) {
    unsigned top = 0;                    // magnitudes compare like their bit patterns, NaN above all
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int d = BLOCK / V / 2; d > 0; d /= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const float t = __uint_as_float(top);
    const bool fine = top < 0x7F800000u, used = fine && t >= SMALLEST;
    const float per_unit = used ? __fmul_rn(127.0f, __frcp_rn(t)) : 0.0f;
    *scale = used ? __fmul_rn(t, 1.0f / 127.0f) : fine ? 0.0f : __int_as_float(0x7FC00000);
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i) w[i / 4] |= (static_cast<unsigned>(__float2int_rn(used ? __fmul_rn(x[i], per_unit) : 0.0f)) & 0xFFu) << (8 * (i % 4));
    *codes = make_uint2(w[0], w[1]);
}

template <int V>
__device__ __forceinline__ void store_codes(int8_t *at, const uint2 &c) {
    if constexpr (V == 8) *reinterpret_cast<uint2 *>(at) = c;
    else *reinterpret_cast<unsigned *>(at) = c.x;
}

template <int V>
__device__ __forceinline__ uint2 load_codes(const int8_t *at) {
    uint2 c = make_uint2(0, 0);
    if constexpr (V == 8) asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(c.x), "=r"(c.y) : "l"(at));
    else asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(c.x) : "l"(at));
    return c;
}

template <int V>
__device__ __forceinline__ void decode(const uint2 &c, float scale, float (&x)[V]) {
    const unsigned w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __fmul_rn(static_cast<float>(static_cast<int>(w[i / 4] << (24 - 8 * (i % 4))) >> 24), scale);
}

__host__ __device__ constexpr int64_t pitch_of(int64_t cols) { return (cols + 15) / 16 * 16; }
__host__ __device__ constexpr int64_t blocks_of(int64_t cols) { return (cols + BLOCK - 1) / BLOCK; }

// ---------------------------------------------------------------------------- sums over a row
// The threads on a row are one warp (several rows to a CTA) or the whole CTA.  `turn` alternates
// between two sets of slots, so that one barrier per sum is enough.
template <bool WARP>
__device__ __forceinline__ float2 row_sum(float2 v, float2 (&slots)[2][GROUP_MAX / 32], int &turn) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, d);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, d);
    }
    if constexpr (!WARP) {
        if (threadIdx.x % 32 == 0) slots[turn][threadIdx.x / 32] = v;
        __syncthreads();
        v = make_float2(0.0f, 0.0f);
        for (unsigned w = 0; w < blockDim.x / 32; ++w) v.x += slots[turn][w].x, v.y += slots[turn][w].y;
        turn ^= 1;
    }
    return v;
}

// --------------------------------------------------------------------------------- layer norm
struct NormParams {
    const void *x, *dout, *weight, *bias;
    void *out;                            // y, or dx
    float *mean, *rstd;                   // written by the forward pass, read by the backward pass
    int8_t *codes;
    float *scales;
    float *parts;                         // backward: partial sums [parts][2][cols]
    void *dweight, *dbias;
    int64_t rows, cols, x_stride, dout_stride, out_stride;
    float eps;
    int param_bf16, n_parts;
};

// y = (x - mean) rstd w + b.  Mean first, then the squared distances from it: both from registers.
template <typename T, bool WIDE, bool WARP, int NV>
__global__ void __launch_bounds__(GROUP_MAX) k_norm_forward(const NormParams p) {
    constexpr int V = Elems<T>::V;
    __shared__ float2 slots[2][GROUP_MAX / 32];
    int turn = 0;
    const int group = WARP ? 32 : blockDim.x, at = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t per_cta = blockDim.x / group, first = blockIdx.x * per_cta + threadIdx.x / group;
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param(p.weight, p.param_bf16, static_cast<int64_t>(at + k * group) * V, p.cols, 1.0f, w[k]);
        load_param(p.bias, p.param_bf16, static_cast<int64_t>(at + k * group) * V, p.cols, 0.0f, b[k]);
    }
    for (int64_t r = first; r < p.rows; r += gridDim.x * per_cta) {
        const T *row = static_cast<const T *>(p.x) + r * p.x_stride;
        float x[NV][V];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            load_row<T, WIDE>(row, static_cast<int64_t>(at + k * group) * V, p.cols, x[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s.x += x[k][i];
        }
        const float mean = row_sum<WARP>(s, slots, turn).x / static_cast<float>(p.cols);
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = WIDE ? static_cast<int64_t>(at + k * group) * V < p.cols : static_cast<int64_t>(at + k * group) * V + i < p.cols;
                x[k][i] = in ? x[k][i] - mean : 0.0f;
                s.x += x[k][i] * x[k][i];
            }
        const float rstd = __frsqrt_rn(row_sum<WARP>(s, slots, turn).x / static_cast<float>(p.cols) + p.eps);
        if (at == 0) {
            if (p.mean != nullptr) p.mean[r] = mean;
            if (p.rstd != nullptr) p.rstd[r] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t col = static_cast<int64_t>(at + k * group) * V;
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] *= rstd;
                y[i] = x[k][i] * w[k][i] + b[k][i];
            }
            store_row<T, WIDE>(static_cast<T *>(p.out) + r * p.out_stride, col, p.cols, y);
            if (p.codes != nullptr) {
                uint2 c;
                float scale;
                encode<V>(x[k], &c, &scale);
                if (col < pitch_of(p.cols)) store_codes<V>(p.codes + r * pitch_of(p.cols) + col, c);
                if (col % BLOCK == 0 && col < p.cols) p.scales[r * blocks_of(p.cols) + col / BLOCK] = scale;
            }
        }
    }
}

// With u = (x - mean) rstd (or its 8-bit checkpoint) and g = dout w:
//   dx = rstd (g - mean(g) - u mean(g u)),  dweight = sum_rows dout u,  dbias = sum_rows dout.
// A CTA goes over rows blockIdx, blockIdx + grid, ... and keeps its columns' sums in registers;
// one row of partial sums per CTA is reduced in a fixed order by k_norm_params: no atomics, so that
// a step gives the same bits when it is run again.
template <typename T, bool WIDE, bool WARP, int NV, bool KEPT>
__global__ void __launch_bounds__(GROUP_MAX) k_norm_backward(const NormParams p) {
    constexpr int V = Elems<T>::V;
    __shared__ float2 slots[2][GROUP_MAX / 32];
    extern __shared__ float joined[];     // WARP: [2][32 * NV * V], the sums of the CTA's warps
    int turn = 0;
    const int group = WARP ? 32 : blockDim.x, at = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t per_cta = blockDim.x / group, first = blockIdx.x * per_cta + threadIdx.x / group;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param(p.weight, p.param_bf16, static_cast<int64_t>(at + k * group) * V, p.cols, 1.0f, w[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.0f;
    }
    const float per_col = 1.0f / static_cast<float>(p.cols);
    for (int64_t r = first; r < p.rows; r += gridDim.x * per_cta) {
        float g[NV][V], u[NV][V];
        const float rstd = p.rstd[r], mean = KEPT ? 0.0f : p.mean[r];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t col = static_cast<int64_t>(at + k * group) * V;
            load_row<T, WIDE>(static_cast<const T *>(p.dout) + r * p.dout_stride, col, p.cols, g[k]);
            if constexpr (KEPT) {
                const bool in = col < p.cols;
                decode<V>(in ? load_codes<V>(p.codes + r * pitch_of(p.cols) + col) : make_uint2(0, 0),
                          in ? p.scales[r * blocks_of(p.cols) + col / BLOCK] : 0.0f, u[k]);
            } else {
                load_row<T, WIDE>(static_cast<const T *>(p.x) + r * p.x_stride, col, p.cols, u[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (!KEPT) u[k][i] = (u[k][i] - mean) * rstd;     // past the row's end g is zero
                dw[k][i] += g[k][i] * u[k][i];
                db[k][i] += g[k][i];
                g[k][i] *= w[k][i];
                s.x += g[k][i];
                s.y += g[k][i] * u[k][i];
            }
        s = row_sum<WARP>(s, slots, turn);
        s.x *= per_col;
        s.y *= per_col;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = (g[k][i] - s.x - u[k][i] * s.y) * rstd;
            store_row<T, WIDE>(static_cast<T *>(p.out) + r * p.out_stride, static_cast<int64_t>(at + k * group) * V, p.cols, y);
        }
    }
    if (p.parts == nullptr) return;
    float *part = p.parts + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
    if constexpr (WARP) {
        constexpr int N = 32 * NV * V;
        for (unsigned turn_of = 0; turn_of < blockDim.x / 32; ++turn_of) {
            if (threadIdx.x / 32 == turn_of) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (at + k * 32) * V + i;
                        joined[c] = turn_of == 0 ? dw[k][i] : joined[c] + dw[k][i];
                        joined[N + c] = turn_of == 0 ? db[k][i] : joined[N + c] + db[k][i];
                    }
            }
            __syncthreads();
        }
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) part[c] = joined[c], part[p.cols + c] = joined[N + c];
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int64_t c = static_cast<int64_t>(at + k * group) * V + i;
                if (c < p.cols) part[c] = dw[k][i], part[p.cols + c] = db[k][i];
            }
    }
}

// Rows too wide for registers: the row is read again for each of its passes (from L2, where a row
// of up to some MB still is), and the column sums come from a kernel of their own.
template <typename T>
__device__ __forceinline__ void load_any(const T *row, int64_t col, int64_t cols, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = col + i < cols ? Elems<T>::up(row[col + i]) : 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(GROUP_MAX) k_norm_forward_any(const NormParams p) {
    __shared__ float2 slots[2][GROUP_MAX / 32];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T *row = static_cast<const T *>(p.x) + r * p.x_stride;
        T *out = static_cast<T *>(p.out) + r * p.out_stride;
        float2 s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) s.x += Elems<T>::up(row[c]);
        const float mean = row_sum<false>(s, slots, turn).x / static_cast<float>(p.cols);
        s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) {
            const float d = Elems<T>::up(row[c]) - mean;
            s.x += d * d;
        }
        const float rstd = __frsqrt_rn(row_sum<false>(s, slots, turn).x / static_cast<float>(p.cols) + p.eps);
        if (threadIdx.x == 0) {
            if (p.mean != nullptr) p.mean[r] = mean;
            if (p.rstd != nullptr) p.rstd[r] = rstd;
        }
        // one block of 128 columns to a warp
        for (int64_t c = static_cast<int64_t>(threadIdx.x) * 4; c < blocks_of(p.cols) * BLOCK; c += blockDim.x * 4) {
            float u[4], w[4], b[4];
            load_any(row, c, p.cols, u);
            load_param(p.weight, p.param_bf16, c, p.cols, 1.0f, w);
            load_param(p.bias, p.param_bf16, c, p.cols, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u[i] = c + i < p.cols ? (u[i] - mean) * rstd : 0.0f;
                if (c + i < p.cols) out[c + i] = Elems<T>::one(u[i] * w[i] + b[i]);
            }
            if (p.codes != nullptr) {
                uint2 codes;
                float scale;
                encode<4>(u, &codes, &scale);
                if (c < pitch_of(p.cols)) store_codes<4>(p.codes + r * pitch_of(p.cols) + c, codes);
                if (c % BLOCK == 0) p.scales[r * blocks_of(p.cols) + c / BLOCK] = scale;
            }
        }
    }
}

// One element of the normalised row, from the row itself or from its checkpoint.
template <typename T, bool KEPT>
__device__ __forceinline__ float unit_at(const NormParams &p, int64_t r, int64_t c, float mean, float rstd) {
    if constexpr (KEPT) return __fmul_rn(static_cast<float>(p.codes[r * pitch_of(p.cols) + c]), p.scales[r * blocks_of(p.cols) + c / BLOCK]);
    else return (Elems<T>::up(static_cast<const T *>(p.x)[r * p.x_stride + c]) - mean) * rstd;
}

template <bool KEPT>
__device__ __forceinline__ float mean_at(const NormParams &p, int64_t r) {
    if constexpr (KEPT) return 0.0f;
    else return p.mean[r];
}

template <typename T, bool KEPT>
__global__ void __launch_bounds__(GROUP_MAX) k_norm_backward_any(const NormParams p) {
    __shared__ float2 slots[2][GROUP_MAX / 32];
    int turn = 0;
    const float per_col = 1.0f / static_cast<float>(p.cols);
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T *dout = static_cast<const T *>(p.dout) + r * p.dout_stride;
        const float rstd = p.rstd[r], mean = mean_at<KEPT>(p, r);
        float2 s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) {
            float w[1];
            load_param(p.weight, p.param_bf16, c, p.cols, 1.0f, w);
            const float g = Elems<T>::up(dout[c]) * w[0];
            s.x += g;
            s.y += g * unit_at<T, KEPT>(p, r, c, mean, rstd);
        }
        s = row_sum<false>(s, slots, turn);
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) {
            float w[1];
            load_param(p.weight, p.param_bf16, c, p.cols, 1.0f, w);
            const float g = Elems<T>::up(dout[c]) * w[0];
            static_cast<T *>(p.out)[r * p.out_stride + c] =
                Elems<T>::one((g - s.x * per_col - unit_at<T, KEPT>(p, r, c, mean, rstd) * (s.y * per_col)) * rstd);
        }
    }
}

// Partial sums of the columns over a range of rows; runs before k_norm_backward_any, whose dx may
// be written over dout.
template <typename T, bool KEPT>
__global__ void k_norm_columns(const NormParams p) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (c >= p.cols) return;
    const int64_t lo = p.rows * blockIdx.y / gridDim.y, hi = p.rows * (blockIdx.y + 1) / gridDim.y;
    float dw = 0.0f, db = 0.0f;
    for (int64_t r = lo; r < hi; ++r) {
        const float d = Elems<T>::up(static_cast<const T *>(p.dout)[r * p.dout_stride + c]);
        dw += d * unit_at<T, KEPT>(p, r, c, mean_at<KEPT>(p, r), p.rstd[r]);
        db += d;
    }
    float *part = p.parts + static_cast<int64_t>(blockIdx.y) * 2 * p.cols;
    part[c] = dw;
    part[p.cols + c] = db;
}

// Sums of the partial rows: 32 columns to a CTA, 16 threads down each, then a tree; blockIdx.y 0
// writes dweight, 1 dbias.  Rounded once, to the parameters' type.
__global__ void __launch_bounds__(512) k_norm_params(const NormParams p) {
    __shared__ float sums[16][33];
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x;
    void *out = blockIdx.y == 0 ? p.dweight : p.dbias;
    if (out == nullptr) return;
    float s = 0.0f;
    if (c < p.cols)
        for (int q = threadIdx.y; q < p.n_parts; q += 16) s += p.parts[(static_cast<int64_t>(q) * 2 + blockIdx.y) * p.cols + c];
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    for (int h = 8; h > 0; h /= 2) {
        if (threadIdx.y < h) sums[threadIdx.y][threadIdx.x] += sums[threadIdx.y + h][threadIdx.x];
        __syncthreads();
    }
    if (threadIdx.y == 0 && c < p.cols) {
        if (p.param_bf16) static_cast<__nv_bfloat16 *>(out)[c] = __float2bfloat16_rn(sums[0][threadIdx.x]);
        else static_cast<float *>(out)[c] = sums[0][threadIdx.x];
    }
}

// ------------------------------------------------------------- activations and checkpoints
// Work is laid out in vectors over rows padded to whole blocks, so that the lanes that hold a block
// are neighbours; every thread takes U vectors, a CTA's width apart.
constexpr int U = 4;
constexpr int THREADS = 256;

struct ElemParams {
    const void *in;                       // x, or dout
    const void *x;                        // backward pass from the rows themselves
    const void *weight, *bias;            // restore
    void *out;
    int8_t *codes;
    float *scales;
    int64_t rows, cols, in_stride, x_stride, out_stride;
    int64_t vectors;                      // rows * per_row
    unsigned per_row;                     // vectors to a padded row
    int param_bf16;
};

// The normal distribution function from Abramowitz and Stegun, formula 7.1.26
// (absolute error of erf below 1.5e-7), with e = exp(-x^2 / 2), which the derivative needs as well.
__device__ __forceinline__ float normal_below(float x, float *e) {
    const float z = fabsf(x) * 0.70710678118654752f;
    const float t = __fdividef(1.0f, fmaf(0.3275911f, z, 1.0f));
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    *e = __expf(-z * z);
    const float tail = 0.5f * q * *e;
    return x < 0.0f ? tail : 1.0f - tail;
}

template <int KIND>
__device__ __forceinline__ float act(float x) {
    if constexpr (KIND == KT_GELU) {
        float e;
        return x * normal_below(x, &e);
    } else {
        return __fdividef(x, 1.0f + __expf(-x));
    }
}

template <int KIND>
__device__ __forceinline__ float slope(float x) {
    if constexpr (KIND == KT_GELU) {
        float e;
        const float below = normal_below(x, &e);
        return fmaf(x * 0.39894228040143268f, e, below);
    } else {
        const float gate = __fdividef(1.0f, 1.0f + __expf(-x));
        return gate * fmaf(x, 1.0f - gate, 1.0f);
    }
}

enum { KIND_NONE = -1 };                  // a checkpoint alone

template <typename T, bool WIDE, int KIND, bool KEEP>
__global__ void __launch_bounds__(THREADS) k_act_forward(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    const int64_t base = static_cast<int64_t>(blockIdx.x) * (U * THREADS) + threadIdx.x;
    float x[U][V];
    int64_t row[U], col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = base + u * THREADS;
        row[u] = i / p.per_row;
        col[u] = (i - row[u] * p.per_row) * V;
        if (i < p.vectors) {
            load_row<T, WIDE>(static_cast<const T *>(p.in) + row[u] * p.in_stride, col[u], p.cols, x[u]);
        } else {
            col[u] = p.per_row * V;       // past every row
#pragma unroll
            for (int j = 0; j < V; ++j) x[u][j] = 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (KIND != KIND_NONE) {
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = act<KIND>(x[u][j]);
            store_row<T, WIDE>(static_cast<T *>(p.out) + row[u] * p.out_stride, col[u], p.cols, y);
        }
        if constexpr (KEEP) {
            uint2 c;
            float scale;
            encode<V>(x[u], &c, &scale);
            if (col[u] < pitch_of(p.cols)) store_codes<V>(p.codes + row[u] * pitch_of(p.cols) + col[u], c);
            if (col[u] % BLOCK == 0 && col[u] < p.cols) p.scales[row[u] * blocks_of(p.cols) + col[u] / BLOCK] = scale;
        }
    }
}

template <typename T, bool WIDE, int KIND, bool KEPT>
__global__ void __launch_bounds__(THREADS) k_act_backward(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    const int64_t base = static_cast<int64_t>(blockIdx.x) * (U * THREADS) + threadIdx.x;
    float x[U][V], d[U][V];
    int64_t row[U], col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = base + u * THREADS;
        row[u] = i / p.per_row;
        col[u] = (i - row[u] * p.per_row) * V;
        if (i < p.vectors && col[u] < p.cols) {
            load_row<T, WIDE>(static_cast<const T *>(p.in) + row[u] * p.in_stride, col[u], p.cols, d[u]);
            if constexpr (KEPT) decode<V>(load_codes<V>(p.codes + row[u] * pitch_of(p.cols) + col[u]), p.scales[row[u] * blocks_of(p.cols) + col[u] / BLOCK], x[u]);
            else load_row<T, WIDE>(static_cast<const T *>(p.x) + row[u] * p.x_stride, col[u], p.cols, x[u]);
        } else {
            col[u] = p.cols;
#pragma unroll
            for (int j = 0; j < V; ++j) x[u][j] = d[u][j] = 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int j = 0; j < V; ++j) d[u][j] *= slope<KIND>(x[u][j]);
        store_row<T, WIDE>(static_cast<T *>(p.out) + row[u] * p.out_stride, col[u], p.cols, d[u]);
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(THREADS) k_restore(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    const int64_t base = static_cast<int64_t>(blockIdx.x) * (U * THREADS) + threadIdx.x;
    float x[U][V];
    int64_t row[U], col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = base + u * THREADS;
        row[u] = i / p.per_row;
        col[u] = (i - row[u] * p.per_row) * V;
        if (i < p.vectors && col[u] < p.cols) {
            decode<V>(load_codes<V>(p.codes + row[u] * pitch_of(p.cols) + col[u]), p.scales[row[u] * blocks_of(p.cols) + col[u] / BLOCK], x[u]);
        } else {
            col[u] = p.cols;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (col[u] >= p.cols) continue;
        if (p.weight != nullptr || p.bias != nullptr) {
            float w[V], b[V];
            load_param(p.weight, p.param_bf16, col[u], p.cols, 1.0f, w);
            load_param(p.bias, p.param_bf16, col[u], p.cols, 0.0f, b);
#pragma unroll
            for (int j = 0; j < V; ++j) x[u][j] = x[u][j] * w[j] + b[j];
        }
        store_row<T, WIDE>(static_cast<T *>(p.out) + row[u] * p.out_stride, col[u], p.cols, x[u]);
    }
}

// ------------------------------------------------------------------------------- host side
int elem_size(int dtype) { return dtype == KT_F32 ? 4 : 2; }

int check_matrix(const char *what, const void *p, int64_t stride, int64_t rows, int64_t cols, int dtype) {
    if (p == nullptr) return fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype)) return fail(KT_ERR_ALIGN, "%s is not element aligned", what);
    if (rows > 1 && stride < cols) return fail(KT_ERR_SHAPE, "%s: row stride %lld below %lld columns", what, (long long)stride, (long long)cols);
    return KT_OK;
}

int check_sizes(int64_t rows, int64_t cols, int dtype) {
    if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_INVALID, "unknown dtype %d", dtype);
    if (rows < 0 || cols < 1 || cols > (1 << 24)) return fail(KT_ERR_SHAPE, "%lld rows of %lld columns: rows >= 0 and 1 <= columns <= 2^24 expected", (long long)rows, (long long)cols);
    if (rows > INT64_C(0x7FFFFFFFFFFF) / cols) return fail(KT_ERR_SHAPE, "%lld x %lld elements are too many", (long long)rows, (long long)cols);
    return KT_OK;
}

int check_codes(const int8_t *codes, const float *scales, bool needed) {
    if (codes == nullptr && scales == nullptr && !needed) return KT_OK;
    if (codes == nullptr || scales == nullptr) return fail(KT_ERR_INVALID, "a checkpoint has codes and scales: one of them is NULL");
    if (reinterpret_cast<uintptr_t>(codes) % 16) return fail(KT_ERR_ALIGN, "codes is not 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(scales) % 4) return fail(KT_ERR_ALIGN, "scales is not 4-byte aligned");
    return KT_OK;
}

int check_params(const void *a, const void *b, int dtype) {
    if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_INVALID, "unknown param_dtype %d", dtype);
    for (const void *p : {a, b})
        if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype)) return fail(KT_ERR_ALIGN, "a parameter is not element aligned");
    return KT_OK;
}

// 128-bit accesses: base and row stride multiples of 16 bytes, whole vectors in a row.
bool wide(const void *p, int64_t stride, int64_t rows, int64_t cols, int dtype) {
    const int64_t es = elem_size(dtype);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols * es % 16 == 0 && (rows <= 1 || stride * es % 16 == 0);
}

int sm_count(int *sms) {
    int dev = 0;
    KT_CUDA(cudaGetDevice(&dev));
    KT_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    return KT_OK;
}

// How the threads share a row: one warp where it can hold the row, else a CTA of up to 512.
struct RowShape {
    bool warp;
    int threads, nv, rows_per_cta;
};
RowShape row_shape(int64_t cols, int dtype) {
    const int v = dtype == KT_F32 ? 4 : 8;
    const int64_t vectors = (pitch_of(cols) + v - 1) / v;
    RowShape s{};
    s.warp = vectors <= 32 * (E / v);
    int group = 32;
    if (!s.warp)
        for (group = 128; group < GROUP_MAX && vectors > static_cast<int64_t>(group) * (E / v);) group *= 2;
    s.threads = s.warp ? 128 : group;
    s.rows_per_cta = s.threads / group;
    s.nv = static_cast<int>((vectors + group - 1) / group);
    if (s.nv == 3) s.nv = 4;
    return s;
}

int64_t norm_parts(int64_t rows, int64_t cols) {
    (void)cols;
    return rows < PARTS_MAX ? rows : PARTS_MAX;
}

template <typename T, bool WIDE, bool WARP, int NV>
void start_norm_forward(const NormParams &p, int grid, int threads, cudaStream_t st) {
    k_norm_forward<T, WIDE, WARP, NV><<<grid, threads, 0, st>>>(p);
}
template <typename T, bool WIDE, bool WARP, int NV>
void start_norm_backward(const NormParams &p, int grid, int threads, cudaStream_t st) {
    const size_t smem = WARP ? 2 * 32 * NV * Elems<T>::V * sizeof(float) : 0;
    if (p.codes != nullptr) k_norm_backward<T, WIDE, WARP, NV, true><<<grid, threads, smem, st>>>(p);
    else k_norm_backward<T, WIDE, WARP, NV, false><<<grid, threads, smem, st>>>(p);
}

template <typename T, bool WIDE, bool WARP>
void start_norm(bool backward, const RowShape &s, const NormParams &p, int grid, cudaStream_t st) {
#define KT_NV(n)                                                                            \
    (backward ? start_norm_backward<T, WIDE, WARP, n>(p, grid, s.threads, st) : start_norm_forward<T, WIDE, WARP, n>(p, grid, s.threads, st))
    if (s.nv == 1) KT_NV(1);
    else if (s.nv == 2) KT_NV(2);
    else if constexpr (E / Elems<T>::V >= 4) KT_NV(4);
#undef KT_NV
}

template <typename T>
void start_norm(bool backward, bool wide_, const RowShape &s, const NormParams &p, int grid, cudaStream_t st) {
    if (wide_) s.warp ? start_norm<T, true, true>(backward, s, p, grid, st) : start_norm<T, true, false>(backward, s, p, grid, st);
    else s.warp ? start_norm<T, false, true>(backward, s, p, grid, st) : start_norm<T, false, false>(backward, s, p, grid, st);
}

template <typename T>
void start_norm_any(bool backward, const NormParams &p, int grid, cudaStream_t st) {
    if (!backward) {
        k_norm_forward_any<T><<<grid, GROUP_MAX, 0, st>>>(p);
        return;
    }
    const dim3 columns(static_cast<unsigned>((p.cols + 127) / 128), p.n_parts);
    if (p.codes != nullptr) {
        if (p.parts != nullptr) k_norm_columns<T, true><<<columns, 128, 0, st>>>(p);
        k_norm_backward_any<T, true><<<grid, GROUP_MAX, 0, st>>>(p);
    } else {
        if (p.parts != nullptr) k_norm_columns<T, false><<<columns, 128, 0, st>>>(p);
        k_norm_backward_any<T, false><<<grid, GROUP_MAX, 0, st>>>(p);
    }
}

int elem_grid(ElemParams *p, int dtype, int64_t *ctas) {
    const int v = dtype == KT_F32 ? 4 : 8;
    p->per_row = static_cast<unsigned>(blocks_of(p->cols) * (BLOCK / v));
    p->vectors = p->rows * p->per_row;
    *ctas = (p->vectors + U * THREADS - 1) / (U * THREADS);
    if (*ctas > INT_MAX) return fail(KT_ERR_SHAPE, "%lld x %lld elements are too many", (long long)p->rows, (long long)p->cols);
    return KT_OK;
}

template <typename T, bool WIDE>
void start_act_forward(const ElemParams &p, int kind, int ctas, cudaStream_t st) {
    const bool keep = p.codes != nullptr;
    if (kind == KT_GELU) keep ? k_act_forward<T, WIDE, KT_GELU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_forward<T, WIDE, KT_GELU, false><<<ctas, THREADS, 0, st>>>(p);
    else if (kind == KT_SILU) keep ? k_act_forward<T, WIDE, KT_SILU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_forward<T, WIDE, KT_SILU, false><<<ctas, THREADS, 0, st>>>(p);
    else k_act_forward<T, WIDE, KIND_NONE, true><<<ctas, THREADS, 0, st>>>(p);
}

template <typename T, bool WIDE>
void start_act_backward(const ElemParams &p, int kind, int ctas, cudaStream_t st) {
    const bool kept = p.codes != nullptr;
    if (kind == KT_GELU) kept ? k_act_backward<T, WIDE, KT_GELU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_backward<T, WIDE, KT_GELU, false><<<ctas, THREADS, 0, st>>>(p);
    else kept ? k_act_backward<T, WIDE, KT_SILU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_backward<T, WIDE, KT_SILU, false><<<ctas, THREADS, 0, st>>>(p);
}

int act_forward(ElemParams p, int dtype, int kind, bool wide_, void *stream) {
    int64_t ctas = 0;
    if (int rc = elem_grid(&p, dtype, &ctas)) return rc;
    if (ctas == 0) return KT_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == KT_F32) wide_ ? start_act_forward<float, true>(p, kind, ctas, st) : start_act_forward<float, false>(p, kind, ctas, st);
    else wide_ ? start_act_forward<__nv_bfloat16, true>(p, kind, ctas, st) : start_act_forward<__nv_bfloat16, false>(p, kind, ctas, st);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

}  // namespace

extern "C" {

int64_t kt_ckpt_pitch(int64_t cols) { return cols < 0 ? 0 : pitch_of(cols); }
int64_t kt_ckpt_blocks(int64_t cols) { return cols < 0 ? 0 : blocks_of(cols); }

int kt_norm_forward(const void *x, int64_t x_stride, const void *weight, const void *bias, int param_dtype, void *out,
                    int64_t out_stride, float *mean, float *rstd, int8_t *codes, float *scales, int64_t rows, int64_t cols,
                    int dtype, float eps, void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (int rc = check_params(weight, bias, param_dtype)) return rc;
    if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(KT_ERR_INVALID, "eps must be finite and not negative");
    if (rows == 0) return KT_OK;
    if (int rc = check_matrix("x", x, x_stride, rows, cols, dtype)) return rc;
    if (int rc = check_matrix("out", out, out_stride, rows, cols, dtype)) return rc;
    if (int rc = check_codes(codes, scales, false)) return rc;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    NormParams p{};
    p.x = x, p.weight = weight, p.bias = bias, p.out = out, p.mean = mean, p.rstd = rstd, p.codes = codes, p.scales = scales;
    p.rows = rows, p.cols = cols, p.x_stride = x_stride, p.out_stride = out_stride, p.eps = eps, p.param_bf16 = param_dtype == KT_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cols > ROW_MAX) {
        const int grid = static_cast<int>(rows < sms * 4 ? rows : sms * 4);
        if (dtype == KT_F32) start_norm_any<float>(false, p, grid, st);
        else start_norm_any<__nv_bfloat16>(false, p, grid, st);
    } else {
        const RowShape s = row_shape(cols, dtype);
        const bool w = wide(x, x_stride, rows, cols, dtype) && wide(out, out_stride, rows, cols, dtype);
        const int64_t need = (rows + s.rows_per_cta - 1) / s.rows_per_cta, most = static_cast<int64_t>(sms) * (1024 / s.threads);
        const int grid = static_cast<int>(need < most ? need : most);
        if (dtype == KT_F32) start_norm<float>(false, w, s, p, grid, st);
        else start_norm<__nv_bfloat16>(false, w, s, p, grid, st);
    }
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

int64_t kt_norm_workspace(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return 0;
    return norm_parts(rows, cols) * 2 * cols * static_cast<int64_t>(sizeof(float));
}

int kt_norm_backward(const void *dout, int64_t dout_stride, const void *x, int64_t x_stride, const float *mean, const int8_t *codes,
                     const float *scales, const float *rstd, const void *weight, int param_dtype, void *dx, int64_t dx_stride,
                     void *dweight, void *dbias, void *workspace, int64_t workspace_bytes, int64_t rows, int64_t cols, int dtype,
                     void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (int rc = check_params(weight, nullptr, param_dtype)) return rc;
    if (int rc = check_params(dweight, dbias, param_dtype)) return rc;
    const bool sums = dweight != nullptr || dbias != nullptr;
    if (rows > 0) {
        if (int rc = check_matrix("dout", dout, dout_stride, rows, cols, dtype)) return rc;
        if (int rc = check_matrix("dx", dx, dx_stride, rows, cols, dtype)) return rc;
        if ((x != nullptr) == (codes != nullptr)) return fail(KT_ERR_INVALID, "either x with mean or codes with scales is needed, not both");
        if (x != nullptr) {
            if (int rc = check_matrix("x", x, x_stride, rows, cols, dtype)) return rc;
            if (mean == nullptr) return fail(KT_ERR_INVALID, "mean is NULL");
        } else if (int rc = check_codes(codes, scales, true)) {
            return rc;
        }
        if (rstd == nullptr) return fail(KT_ERR_INVALID, "rstd is NULL");
        if (sums) {
            const int64_t need = kt_norm_workspace(rows, cols);
            if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
            if (workspace_bytes < need) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)workspace_bytes, (long long)need);
            if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
        }
    }
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    NormParams p{};
    p.dout = dout, p.x = x, p.weight = weight, p.out = dx, p.mean = const_cast<float *>(mean), p.rstd = const_cast<float *>(rstd);
    p.codes = const_cast<int8_t *>(codes), p.scales = const_cast<float *>(scales), p.dweight = dweight, p.dbias = dbias;
    p.parts = sums ? static_cast<float *>(workspace) : nullptr;
    p.rows = rows, p.cols = cols, p.dout_stride = dout_stride, p.x_stride = x_stride, p.out_stride = dx_stride, p.param_bf16 = param_dtype == KT_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows > 0 && cols > ROW_MAX) {
        p.n_parts = static_cast<int>(rows < 16 ? rows : 16);
        const int grid = static_cast<int>(rows < sms * 4 ? rows : sms * 4);
        if (dtype == KT_F32) start_norm_any<float>(true, p, grid, st);
        else start_norm_any<__nv_bfloat16>(true, p, grid, st);
        KT_CUDA(cudaGetLastError());
    } else if (rows > 0) {
        const RowShape s = row_shape(cols, dtype);
        const bool w = wide(dout, dout_stride, rows, cols, dtype) && wide(dx, dx_stride, rows, cols, dtype) && (x == nullptr || wide(x, x_stride, rows, cols, dtype));
        const int64_t need = (rows + s.rows_per_cta - 1) / s.rows_per_cta;
        const int64_t busy = static_cast<int64_t>(sms) * (512 / s.threads), most = busy < norm_parts(rows, cols) ? busy : norm_parts(rows, cols);
        p.n_parts = static_cast<int>(need < most ? need : most);
        if (dtype == KT_F32) start_norm<float>(true, w, s, p, p.n_parts, st);
        else start_norm<__nv_bfloat16>(true, w, s, p, p.n_parts, st);
        KT_CUDA(cudaGetLastError());
    }
    if (sums) {
        k_norm_params<<<dim3(static_cast<unsigned>((cols + 31) / 32), 2), dim3(32, 16), 0, st>>>(p);
        KT_CUDA(cudaGetLastError());
    }
    return KT_OK;
}

int kt_ckpt_store(const void *x, int64_t x_stride, int8_t *codes, float *scales, int64_t rows, int64_t cols, int dtype, void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (rows == 0) return KT_OK;
    if (int rc = check_matrix("x", x, x_stride, rows, cols, dtype)) return rc;
    if (int rc = check_codes(codes, scales, true)) return rc;
    ElemParams p{};
    p.in = x, p.in_stride = x_stride, p.codes = codes, p.scales = scales, p.rows = rows, p.cols = cols;
    return act_forward(p, dtype, KIND_NONE, wide(x, x_stride, rows, cols, dtype), stream);
}

int kt_ckpt_restore(const int8_t *codes, const float *scales, const void *weight, const void *bias, int param_dtype, void *out,
                    int64_t out_stride, int64_t rows, int64_t cols, int dtype, void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (int rc = check_params(weight, bias, param_dtype)) return rc;
    if (rows == 0) return KT_OK;
    if (int rc = check_codes(codes, scales, true)) return rc;
    if (int rc = check_matrix("out", out, out_stride, rows, cols, dtype)) return rc;
    ElemParams p{};
    p.codes = const_cast<int8_t *>(codes), p.scales = const_cast<float *>(scales), p.weight = weight, p.bias = bias;
    p.param_bf16 = param_dtype == KT_BF16, p.out = out, p.out_stride = out_stride, p.rows = rows, p.cols = cols;
    int64_t ctas = 0;
    if (int rc = elem_grid(&p, dtype, &ctas)) return rc;
    const bool w = wide(out, out_stride, rows, cols, dtype);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == KT_F32) w ? k_restore<float, true><<<ctas, THREADS, 0, st>>>(p) : k_restore<float, false><<<ctas, THREADS, 0, st>>>(p);
    else w ? k_restore<__nv_bfloat16, true><<<ctas, THREADS, 0, st>>>(p) : k_restore<__nv_bfloat16, false><<<ctas, THREADS, 0, st>>>(p);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

int kt_act_forward(const void *x, int64_t x_stride, void *out, int64_t out_stride, int8_t *codes, float *scales, int64_t rows,
                   int64_t cols, int dtype, int kind, void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (kind != KT_GELU && kind != KT_SILU) return fail(KT_ERR_INVALID, "unknown activation %d", kind);
    if (rows == 0) return KT_OK;
    if (int rc = check_matrix("x", x, x_stride, rows, cols, dtype)) return rc;
    if (int rc = check_matrix("out", out, out_stride, rows, cols, dtype)) return rc;
    if (int rc = check_codes(codes, scales, false)) return rc;
    ElemParams p{};
    p.in = x, p.in_stride = x_stride, p.out = out, p.out_stride = out_stride, p.codes = codes, p.scales = scales, p.rows = rows, p.cols = cols;
    return act_forward(p, dtype, kind, wide(x, x_stride, rows, cols, dtype) && wide(out, out_stride, rows, cols, dtype), stream);
}

int kt_act_backward(const void *dout, int64_t dout_stride, const void *x, int64_t x_stride, const int8_t *codes, const float *scales,
                    void *dx, int64_t dx_stride, int64_t rows, int64_t cols, int dtype, int kind, void *stream) {
    if (int rc = check_sizes(rows, cols, dtype)) return rc;
    if (kind != KT_GELU && kind != KT_SILU) return fail(KT_ERR_INVALID, "unknown activation %d", kind);
    if (rows == 0) return KT_OK;
    if (int rc = check_matrix("dout", dout, dout_stride, rows, cols, dtype)) return rc;
    if (int rc = check_matrix("dx", dx, dx_stride, rows, cols, dtype)) return rc;
    if ((x != nullptr) == (codes != nullptr)) return fail(KT_ERR_INVALID, "either x or codes with scales is needed, not both");
    if (x != nullptr) {
        if (int rc = check_matrix("x", x, x_stride, rows, cols, dtype)) return rc;
    } else if (int rc = check_codes(codes, scales, true)) {
        return rc;
    }
    ElemParams p{};
    p.in = dout, p.in_stride = dout_stride, p.x = x, p.x_stride = x_stride, p.out = dx, p.out_stride = dx_stride;
    p.codes = const_cast<int8_t *>(codes), p.scales = const_cast<float *>(scales), p.rows = rows, p.cols = cols;
    int64_t ctas = 0;
    if (int rc = elem_grid(&p, dtype, &ctas)) return rc;
    const bool w = wide(dout, dout_stride, rows, cols, dtype) && wide(dx, dx_stride, rows, cols, dtype) && (x == nullptr || wide(x, x_stride, rows, cols, dtype));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == KT_F32) w ? start_act_backward<float, true>(p, kind, ctas, st) : start_act_backward<float, false>(p, kind, ctas, st);
    else w ? start_act_backward<__nv_bfloat16, true>(p, kind, ctas, st) : start_act_backward<__nv_bfloat16, false>(p, kind, ctas, st);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

}  // extern "C"
