// kt_rows.cu -- operators on rows of activations that a data-parallel worker runs to obtain the
// gradients the library synchronises: layer norm forward and backward (with the reduction of the
// weight's and the bias' gradient over all rows), GELU / SiLU forward and backward, and the 8-bit
// checkpoints that both can leave for the backward pass.  Contracts: include/kaitian.h.
//
// Memory sets the floor of all of it: a row is read once with 128-bit loads, stays in registers as fp32
// for its statistics and its result, and is written once.  Rows whose address or width does not
// allow 128-bit accesses take the same kernels with narrower accesses (template argument WIDE), rows
// of layer norm above ROW_MAX columns kernels of their own; instructions bound these, and layer norm with checkpoints.
//
// 8-bit checkpoints.  A block of KT_CKPT_BLOCK = 128 columns of a row shares one fp32 scale:
//   top = max |x|,  scale = top / 127,  code = rint(x * 127 / top) in -127 ... 127,
// so that a value is off by at most scale / 2.  A block with top < 2^-100 is kept as zeros (127 / top
// must not overflow); one with an infinity or a NaN gets scale NaN, so that it restores as NaN
// and is not silently cut off.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <climits>
#include <cmath>

#include "kt_internal.h"
#include "kt_pairs.cuh"

using namespace ktd;

namespace {

constexpr int BLOCK = KT_CKPT_BLOCK;
constexpr int E = 16;                    // row elements that a thread keeps in registers
constexpr int GROUP_MAX = 512;           // threads on one row at most
constexpr int64_t ROW_MAX = E * GROUP_MAX;   // wider rows are read again instead of kept
constexpr int SMS = 148;                 // of a B200: the grids are cut to them
constexpr float SMALLEST = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Maximum and minimum that keep a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float inverse_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Copies into shared memory that the issuing thread alone waits for and reads again.
template <int BYTES>
__device__ __forceinline__ void copy_ahead(void *to, const void *from) {
    const unsigned at = static_cast<unsigned>(__cvta_generic_to_shared(to));
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

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

// One vector of a row as it lies in memory; columns at or past `cols` are zeros.
template <typename T, bool WIDE>
__device__ __forceinline__ uint4 load_row(const T *row, int64_t col, int64_t cols) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if constexpr (WIDE) {
        if (col < cols) r = load16(row + col);
    } else if constexpr (sizeof(T) == 4) {
        const unsigned *at = reinterpret_cast<const unsigned *>(row) + col;
        if (col < cols) r.x = at[0];
        if (col + 1 < cols) r.y = at[1];
        if (col + 2 < cols) r.z = at[2];
        if (col + 3 < cols) r.w = at[3];
    } else {
        // whole words, of which the first and the last may be shared with other rows: half as many loads as elements
        const unsigned off = reinterpret_cast<uintptr_t>(row + col) & 2;
        const unsigned *at = reinterpret_cast<const unsigned *>(reinterpret_cast<const char *>(row + col) - off);
        const int left = static_cast<int>(cols - col > 8 ? 16 : (cols - col) * 2), end = left + static_cast<int>(off);       // bytes wanted, and where they end
        unsigned w[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = left > 0 && 4 * i < end ? at[i] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __funnelshift_r(w[i], w[i + 1], off * 8);
            if (left < 4 * i + 4) w[i] = left <= 4 * i ? 0 : w[i] & 0xFFFFu;
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}

// Rows of bf16 that are not made of aligned vectors are written in aligned 16-byte pieces all the same: a lane
// writes the piece in which its vector starts, with the end of its left neighbour's vector in it (the lanes of
// a warp hold vectors that follow one another, and all of them call); what no lane can write as a
// whole piece goes in aligned parts of 8, 4 and 2 bytes, and at the row's end element by element.
template <typename T, bool WIDE>
__device__ __forceinline__ void store_row(T *row, int64_t col, int64_t cols, const float (&x)[Elems<T>::V]) {
    constexpr int V = Elems<T>::V;
    const uint4 r = Elems<T>::narrow(x);
    if constexpr (WIDE) {
        if (col < cols) *reinterpret_cast<uint4 *>(row + col) = r;
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col + i < cols) row[col + i] = x[i];
    } else {
        const unsigned off = reinterpret_cast<uintptr_t>(row + col) & 15;
        const int first = 16 - static_cast<int>(off);                                   // bytes in the first piece
        const int64_t left = (cols - col) * static_cast<int64_t>(sizeof(T));
        uint4 l;
        l.x = __shfl_up_sync(0xFFFFFFFFu, r.x, 1), l.y = __shfl_up_sync(0xFFFFFFFFu, r.y, 1);
        l.z = __shfl_up_sync(0xFFFFFFFFu, r.z, 1), l.w = __shfl_up_sync(0xFFFFFFFFu, r.w, 1);
        if (left <= 0) return;
        const bool whole = left >= first && (off == 0 || (threadIdx.x % 32 > 0 && col > 0));
        if (whole) {
            unsigned w[8] = {l.x, l.y, l.z, l.w, r.x, r.y, r.z, r.w};                  // bytes 16 - off ... 32 - off of the two
            if (first & 16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = w[i + 4];
            } else {
                if (first & 8) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                }
                if (first & 4) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                }
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (first & 2) * 8);
                }
            }
            *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(row + col) - off) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        // the right neighbour takes the end along if it writes a whole piece
        const bool taken = off == 0 || (threadIdx.x % 32 < 31 && left - 16 >= first);
        if (whole && taken) return;
        char *const to = reinterpret_cast<char *>(row + col);
        if (left < 16) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (2 * i < left && (2 * i < first ? !whole : !taken)) row[col + i] = Elems<T>::one(x[i]);
            return;
        }
        const bool odd = off & 2;
        if (!whole) {                                // `first` bytes, up to a multiple of 16: 2, 4, 8 of them
            if (odd) *reinterpret_cast<unsigned short *>(to) = static_cast<unsigned short>(r.x);
            const unsigned w[3] = {odd ? __funnelshift_r(r.x, r.y, 16) : r.x, odd ? __funnelshift_r(r.y, r.z, 16) : r.y, odd ? __funnelshift_r(r.z, r.w, 16) : r.z};
            char *const at = to + (off & 2);
            if (first & 4) *reinterpret_cast<unsigned *>(at) = w[0];
            if (first & 8) *reinterpret_cast<uint2 *>(at + (first & 4)) = first & 4 ? make_uint2(w[1], w[2]) : make_uint2(w[0], w[1]);
        }
        if (!taken) {                                // the last `off` bytes, from a multiple of 16 on: 8, 4, 2 of them
            const unsigned w[3] = {odd ? __funnelshift_r(r.x, r.y, 16) : r.y, odd ? __funnelshift_r(r.y, r.z, 16) : r.z, odd ? __funnelshift_r(r.z, r.w, 16) : r.w};
            if (off & 8) *reinterpret_cast<uint2 *>(to + first) = off & 4 ? make_uint2(w[0], w[1]) : make_uint2(w[1], w[2]);
            if (off & 4) *reinterpret_cast<unsigned *>(to + 12 - (off & 2)) = w[2];
            if (odd) *reinterpret_cast<unsigned short *>(to + 14) = static_cast<unsigned short>(r.w >> 16);
        }
    }
}

// V columns of a weight or bias (fp32 or bf16, any alignment); `missing` where there is none.
template <int V>
__device__ __forceinline__ void load_param(const void *p, bool bf16, int64_t col, int64_t cols, float missing, float (&w)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = missing;
    if (p == nullptr || col >= cols) return;
    if (!bf16 && V >= 4 && col + V <= cols && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
        for (int i = 0; i + 3 < V; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + col + i);
            w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (col + i < cols) w[i] = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[col + i]) : static_cast<const float *>(p)[col + i];
}

__device__ __forceinline__ void store_param(void *p, bool bf16, int64_t col, float x) {
    if (p == nullptr) return;
    if (bf16) static_cast<__nv_bfloat16 *>(p)[col] = __float2bfloat16_rn(x);
    else static_cast<float *>(p)[col] = x;
}

// The V codes of one vector and the scale of its block.  The 128 / V lanes that hold a block are
// neighbours; all lanes of the warp call it, those without columns of the row with `in` false.  Columns
// past the row's end in a vector that has some hold zeros.  Adding 1.5 * 2^23
// rounds to the nearest whole number and leaves it, as a signed byte, in the sum's lowest bits.
template <int V>
__device__ __forceinline__ void encode(const float (&x)[V], bool in, uint2 *codes, float *scale) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) top = max_nan(top, fabsf(x[i]));
    if (!in) top = 0.0f;
#pragma unroll
    for (int d = BLOCK / V / 2; d > 0; d /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const bool fine = top < INFINITY, used = fine && top >= SMALLEST;
    const float per_unit = used ? __fmul_rn(127.0f, __frcp_rn(top)) : 0.0f;
    *scale = used ? __fmul_rn(top, 1.0f / 127.0f) : fine ? 0.0f : __int_as_float(0x7FC00000);
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        unsigned q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = __float_as_uint(__fadd_rn(__fmul_rn(x[i + j], per_unit), 12582912.0f));       // two roundings, not one
        const unsigned lo = __byte_perm(q[0], q[1], 0x0040), hi = __byte_perm(q[2], q[3], 0x0040);
        w[i / 4] = __byte_perm(lo, hi, 0x5410);
    }
    *codes = in ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
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

// A byte c + 128 in the lowest bits of 2^23 is 2^23 + 128 + c as a float.
template <int V>
__device__ __forceinline__ void decode(const uint2 &c, float scale, float (&x)[V]) {
    const unsigned w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float2 f = make_float2(__uint_as_float(__byte_perm(w[i / 4], 0x4B000000u, 0x7440 + i % 4)), __uint_as_float(__byte_perm(w[i / 4], 0x4B000000u, 0x7440 + i % 4 + 1)));
        const float2 v = mul2(add2(f, both(-8388736.0f)), both(scale));
        x[i] = v.x, x[i + 1] = v.y;
    }
}

__host__ __device__ constexpr int64_t pitch_of(int64_t cols) { return (cols + 15) / 16 * 16; }
__host__ __device__ constexpr int64_t blocks_of(int64_t cols) { return (cols + BLOCK - 1) / BLOCK; }

// The sum over a CTA of two values.  `turn` alternates between two sets of slots, so that one barrier
// per sum is enough.
__device__ __forceinline__ float2 cta_sum(float2 v, float2 (&slots)[2][GROUP_MAX / 32], int &turn) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, d);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, d);
    }
    if (threadIdx.x % 32 == 0) slots[turn][threadIdx.x / 32] = v;
    __syncthreads();
    v = make_float2(0.0f, 0.0f);
    for (unsigned w = 0; w < blockDim.x / 32; ++w) v.x += slots[turn][w].x, v.y += slots[turn][w].y;
    turn ^= 1;
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
    int param_bf16, n_parts, joint;       // joint: the backward pass' CTAs are one cluster
};

// The threads on a row are a warp or a group of 64 to 512 (GROUPS_OF_ROW); forward, a CTA is a group, or four
// warps, backward as many groups as 512 threads hold.  A thread takes the
// vectors at, at + GROUP, ... of its row.  A CTA goes over rows blockIdx, blockIdx + grid, ... and keeps
// its columns' weights (and, backward, their sums) in registers.  Where rows allow 128-bit accesses the
// rows to come are copied into shared memory ahead of their turn, AHEAD of them at a time, each thread
// its own vectors: the copies are in flight while the sums over the current row are formed, and only
// these need a barrier.
// (Three rows ahead; two where a row and its gradient take 64 KB for the threads of an SM.)
template <int NV>
__host__ __device__ constexpr int rows_ahead() { return NV >= 4 ? 2 : 3; }

template <int GROUP>
__host__ __device__ constexpr int norm_threads() { return GROUP == 32 ? 128 : GROUP; }

template <int GROUP>
__host__ __device__ constexpr int backward_threads() { return GROUP_MAX / GROUP * GROUP; }

// Threads on an SM in the forward pass: as many as the registers of 16 elements to a thread allow.
__host__ __device__ constexpr int forward_threads(int elements) { return elements == E ? 640 : 768; }

// Waits for the threads on a row; a CTA with several rows has a barrier for each.
template <int GROUP>
__device__ __forceinline__ void group_barrier(int group) {
    asm volatile("barrier.sync %0, %1;" ::"r"(group + 1), "n"(GROUP) : "memory");
}

template <int GROUP, int NV, int V>
__device__ __forceinline__ int column(int at, int k) { return (at + k * GROUP) * V; }

// Rows of bf16 whose vectors do not start at multiples of 16 bytes are copied ahead as well, in the aligned pieces that hold
// them: a lane copies the piece in which its vector starts, the last one that behind too, and a vector is put together
// from two pieces.  (The ends of a row's first and last piece belong to others and are not looked at.)  Against loads
// by words, a row ahead in the forward pass only: 125 instead of 147 us for the backward pass on 8192 x 5669, 52 instead of 59 for
// the forward pass on 16384 x 1111.  What is left there is the vectors' assembly and the stores (store_row).
// Rows of fp32 take loads by elements.
template <typename T, bool WIDE>
__host__ __device__ constexpr bool in_ring() { return WIDE || sizeof(T) == 2; }
template <bool WIDE>
__host__ __device__ constexpr int cells_of_warp() { return WIDE ? 32 : 33; }
template <bool WIDE, int THREADS>
__device__ __forceinline__ int cell_of(int set) { return (set * (THREADS / 32) + threadIdx.x / 32) * cells_of_warp<WIDE>() + threadIdx.x % 32; }

template <typename T, bool WIDE>
__device__ __forceinline__ void copy_vector(uint4 *to, const T *row, int col, int cols) {
    if constexpr (WIDE) {
        if (col < cols) copy_ahead<16>(to, row + col);
    } else {
        const uintptr_t from = reinterpret_cast<uintptr_t>(row + col) & ~static_cast<uintptr_t>(15), end = reinterpret_cast<uintptr_t>(row + cols);
        if (from < end) copy_ahead<16>(to, reinterpret_cast<const void *>(from));
        if (threadIdx.x % 32 == 31 && from + 16 < end) copy_ahead<16>(to + 1, reinterpret_cast<const void *>(from + 16));
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ uint4 take_vector(const uint4 *from, const T *row, int col, int cols) {
    if (col >= cols) return make_uint4(0, 0, 0, 0);
    if constexpr (WIDE) return *from;
    const unsigned off = reinterpret_cast<uintptr_t>(row) & 15;        // where the vector starts in its piece
    const unsigned *const words = reinterpret_cast<const unsigned *>(from) + off / 4;
    unsigned w[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = words[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (off & 2) * 8);
    const int left = (cols - col) * static_cast<int>(sizeof(T));
    if (left < 16)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (left < 4 * i + 4) w[i] = left <= 4 * i ? 0 : w[i] & 0xFFFFu;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// y = (x - mean) rstd w + b.  A warp takes the mean of its part of the row and the squares around that
// mean; the parts are joined with the exact formula for two samples, so that one barrier is enough
// and nothing cancels.  Bound by memory: 16384 x 4096 bf16 in 53 us (5080 GB/s; a plain copy reaches 6530); with the
// checkpoint by instructions (2.4 a cycle, DRAM at 43 % of its cycles): 73 us, 4600 GB/s.  64 x 512 in 2.8 us, a launch.
template <typename T, bool WIDE, int GROUP, int NV>
__global__ void __launch_bounds__(norm_threads<GROUP>(), forward_threads(NV * Elems<T>::V) / norm_threads<GROUP>()) k_norm_forward(const NormParams p) {
    constexpr int V = Elems<T>::V, THREADS = norm_threads<GROUP>(), WARPS = GROUP / 32, AHEAD = rows_ahead<NV>();
    constexpr bool RING = in_ring<T, WIDE>();
    extern __shared__ uint4 ring[];              // RING: [AHEAD + 1][NV][THREADS / 32][cells_of_warp]
    __shared__ float2 slots[2][WARPS];
    __shared__ float counts[WARPS];
    const int at = threadIdx.x % GROUP;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (THREADS / GROUP), first = static_cast<int64_t>(blockIdx.x) * (THREADS / GROUP) + threadIdx.x / GROUP;
    const int cols = static_cast<int>(p.cols), pitch = static_cast<int>(pitch_of(cols)), blocks = static_cast<int>(blocks_of(cols));
    const float per_col = 1.0f / static_cast<float>(cols);
    auto slot = [&](int stage, int k) { return ring + cell_of<WIDE, THREADS>(stage * NV + k); };
    auto fetch = [&](int64_t r, int stage) {
        if (r < p.rows)
#pragma unroll
            for (int k = 0; k < NV; ++k) copy_vector<T, WIDE>(slot(stage, k), static_cast<const T *>(p.x) + r * p.x_stride, column<GROUP, NV, V>(at, k), cols);
        copies_issued();
    };
    auto part_of = [&](int warp) {               // elements of the row that a warp holds
        int n = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) n += min(max(cols - column<GROUP, NV, V>(warp * 32, k), 0), 32 * V);
        return static_cast<float>(n);
    };
    uint4 raw[NV];
    if constexpr (RING) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) fetch(first + s * step, s);
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) raw[k] = first < p.rows ? load_row<T, WIDE>(static_cast<const T *>(p.x) + first * p.x_stride, column<GROUP, NV, V>(at, k), cols) : make_uint4(0, 0, 0, 0);
    }
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param(p.weight, p.param_bf16, column<GROUP, NV, V>(at, k), cols, 1.0f, w[k]);
        load_param(p.bias, p.param_bf16, column<GROUP, NV, V>(at, k), cols, 0.0f, b[k]);
    }
    const float mine = part_of(at / 32), per_mine = mine > 0.0f ? 1.0f / mine : 0.0f;
    if (WARPS > 1 && threadIdx.x % 32 == 0) counts[at / 32] = mine;     // read after the first row's barrier
    int stage = 0, turn = 0;
    for (int64_t r = first; r < p.rows; r += step) {
        float x[NV][V];
        float2 s = both(0.0f);
        if constexpr (RING) {
            wait_copies<AHEAD - 1>();
            if constexpr (!WIDE) __syncwarp();       // lanes read their neighbours' pieces
#pragma unroll
            for (int k = 0; k < NV; ++k) raw[k] = take_vector<T, WIDE>(slot(stage, k), static_cast<const T *>(p.x) + r * p.x_stride, column<GROUP, NV, V>(at, k), cols);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            Elems<T>::widen(raw[k], x[k]);
#pragma unroll
            for (int i = 0; i < V; i += 2) s = add2(s, make_float2(x[k][i], x[k][i + 1]));
        }
        if constexpr (RING) {
            fetch(r + AHEAD * step, stage == 0 ? AHEAD : stage - 1);
            stage = stage == AHEAD ? 0 : stage + 1;
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (r + step < p.rows) raw[k] = load_row<T, WIDE>(static_cast<const T *>(p.x) + (r + step) * p.x_stride, column<GROUP, NV, V>(at, k), cols);
        }
        float mean = s.x + s.y;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, d);
        mean *= per_mine;
        float2 sq = both(0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = column<GROUP, NV, V>(at, k);
            if (col >= cols) continue;
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                float2 d = add2(make_float2(x[k][i], x[k][i + 1]), both(-mean));
                if (!WIDE && col + i >= cols) d.x = 0.0f;
                if (!WIDE && col + i + 1 >= cols) d.y = 0.0f;
                sq = fma2(d, d, sq);
            }
        }
        float m2 = sq.x + sq.y;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) m2 += __shfl_xor_sync(0xFFFFFFFFu, m2, d);
        if constexpr (WARPS > 1) {
            if (threadIdx.x % 32 == 0) slots[turn][at / 32] = make_float2(mean, m2);
            __syncthreads();
            mean = m2 = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) mean += counts[i] * slots[turn][i].x;
            mean *= per_col;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float2 part = slots[turn][i];
                m2 += fmaf(counts[i] * (part.x - mean), part.x - mean, part.y);
            }
            turn ^= 1;
        }
        const float rstd = __frsqrt_rn(m2 * per_col + p.eps);
        if (at == 0) {
            if (p.mean != nullptr) p.mean[r] = mean;
            if (p.rstd != nullptr) p.rstd[r] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = column<GROUP, NV, V>(at, k);
            float y[V];
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const float2 u = mul2(add2(make_float2(x[k][i], x[k][i + 1]), both(-mean)), both(rstd));
                const float2 v = fma2(u, make_float2(w[k][i], w[k][i + 1]), make_float2(b[k][i], b[k][i + 1]));
                x[k][i] = u.x, x[k][i + 1] = u.y, y[i] = v.x, y[i + 1] = v.y;
            }
            store_row<T, WIDE>(static_cast<T *>(p.out) + r * p.out_stride, col, cols, y);
            if (p.codes != nullptr) {
                uint2 c;
                float scale;
                if constexpr (!WIDE)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (col + i >= cols) x[k][i] = 0.0f;
                encode<V>(x[k], col < cols, &c, &scale);
                if (col < pitch) store_codes<V>(p.codes + r * pitch + col, c);
                if (col % BLOCK == 0 && col < cols) p.scales[r * blocks + col / BLOCK] = scale;
            }
        }
    }
}

// With u = (x - mean) rstd (or its 8-bit checkpoint) and g = dout w:
//   dx = rstd (g - mean(g) - u mean(g u)),  dweight = sum_rows dout u,  dbias = sum_rows dout.
// A CTA of up to 512 threads fills an SM's registers; its groups join their columns' sums at the end.  With few rows the CTAs
// are one cluster that joins its sums through distributed shared memory; else one row of partial
// sums per CTA is reduced in a fixed order by k_norm_params: no atomics either way, so that a step gives the same bits
// when it is run again.  (With a CTA to a group, four times as many partial sums: 47.6 instead of 38.6 us for
// 16384 x 2048 bf16 from a checkpoint.)  Bound by memory where rows are many: 16384 x 4096 bf16 in 69 us (5830 GB/s); from
// a checkpoint by instructions (2.2 a cycle, DRAM 43 %): 16384 x 2048 in 38 us (4400 GB/s); 4999 x 1000 fp32 in 16, some 4 of
// them the second kernel's.
template <typename T, bool WIDE, int GROUP, int NV, bool KEPT>
__global__ void __launch_bounds__(backward_threads<GROUP>(), 1) k_norm_backward(const NormParams p) {
    constexpr int V = Elems<T>::V, THREADS = backward_threads<GROUP>(), GROUPS = THREADS / GROUP, WARPS = GROUP / 32, AHEAD = rows_ahead<NV>();
    constexpr int SOURCE = KEPT ? V : 16;        // bytes of a vector of u: codes, or x itself
    // RING: [AHEAD + 1][NV][THREADS / 32][cells_of_warp] vectors of dout, then as many of SOURCE bytes, then (KEPT) scales;
    // afterwards the sums of the CTA's groups
    extern __shared__ uint4 ring[];
    __shared__ float2 slots[GROUPS][2][WARPS];
    constexpr bool RING = in_ring<T, WIDE>();
    constexpr int CELLS = (AHEAD + 1) * NV * (THREADS / 32) * cells_of_warp<WIDE>();
    char *const ring_u = reinterpret_cast<char *>(ring + CELLS);
    float *const ring_s = reinterpret_cast<float *>(ring_u + CELLS * SOURCE);
    const int at = threadIdx.x % GROUP, group = threadIdx.x / GROUP;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (THREADS / GROUP), first = static_cast<int64_t>(blockIdx.x) * (THREADS / GROUP) + threadIdx.x / GROUP;
    const int cols = static_cast<int>(p.cols), pitch = static_cast<int>(pitch_of(cols)), blocks = static_cast<int>(blocks_of(cols));
    const float per_col = 1.0f / static_cast<float>(cols);
    let_next_begin();
    // Whether any of a warp's k-th vectors lies in the row.  (From a checkpoint, which leaves less to do for a vector, the
    // branches cost more than they save in full rows: 39.4 against 37.9 us for 16384 x 2048; from x they save even there,
    // 69 against 74 for 16384 x 4096.)
    auto some = [&](int k) { return KEPT || k == 0 || column<GROUP, NV, V>(at & ~31, k) < cols; };
    auto cell = [&](int stage, int k) { return cell_of<WIDE, THREADS>(stage * NV + k); };
    auto dout_at = [&](int64_t r) { return static_cast<const T *>(p.dout) + r * p.dout_stride; };
    auto x_at = [&](int64_t r) { return static_cast<const T *>(p.x) + r * p.x_stride; };
    auto codes_at = [&](int64_t r, int k) { return p.codes + r * pitch + column<GROUP, NV, V>(at, k); };
    auto scale_at = [&](int64_t r, int k) { return p.scales + r * blocks + column<GROUP, NV, V>(at, k) / BLOCK; };
    auto fetch = [&](int64_t r, int stage) {
        if (r < p.rows)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (!some(k)) continue;
                const int c = cell(stage, k), col = column<GROUP, NV, V>(at, k);
                copy_vector<T, WIDE>(ring + c, dout_at(r), col, cols);
                if constexpr (!KEPT) {
                    copy_vector<T, WIDE>(reinterpret_cast<uint4 *>(ring_u) + c, x_at(r), col, cols);
                } else if (col < cols) {
                    copy_ahead<SOURCE>(ring_u + c * SOURCE, codes_at(r, k));
                    copy_ahead<4>(ring_s + c, scale_at(r, k));
                }
            }
        copies_issued();
    };
    if constexpr (RING) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) fetch(first + s * step, s);
    }
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_param(p.weight, p.param_bf16, column<GROUP, NV, V>(at, k), cols, 1.0f, w[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.0f;
    }
    float rstd = first < p.rows ? p.rstd[first] : 0.0f, mean = !KEPT && first < p.rows ? p.mean[first] : 0.0f;
    int stage = 0, turn = 0;
    for (int64_t r = first; r < p.rows; r += step) {
        float g[NV][V], u[NV][V];
        float2 s1 = both(0.0f), s2 = both(0.0f);
        if constexpr (RING) wait_copies<AHEAD - 1>();
        if constexpr (RING && !WIDE) __syncwarp();       // lanes read their neighbours' pieces
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!some(k)) continue;
            const int c = cell(stage, k), col = column<GROUP, NV, V>(at, k);
            const bool in = col < cols;
            Elems<T>::widen(RING ? take_vector<T, WIDE>(ring + c, dout_at(r), col, cols) : load_row<T, WIDE>(dout_at(r), col, cols), g[k]);
            if constexpr (KEPT) {
                uint2 codes = make_uint2(0, 0);
                float scale = 0.0f;
                if constexpr (RING) {
                    if (in) {
                        if constexpr (V == 8) codes = *reinterpret_cast<const uint2 *>(ring_u + c * SOURCE);
                        else codes.x = *reinterpret_cast<const unsigned *>(ring_u + c * SOURCE);
                        scale = ring_s[c];
                    }
                } else if (in) {
                    codes = load_codes<V>(codes_at(r, k));
                    scale = *scale_at(r, k);
                }
                decode<V>(codes, scale, u[k]);
            } else {
                Elems<T>::widen(RING ? take_vector<T, WIDE>(reinterpret_cast<const uint4 *>(ring_u) + c, x_at(r), col, cols) : load_row<T, WIDE>(x_at(r), col, cols), u[k]);
            }
        }
        const float by = rstd, shift = mean;
        if constexpr (RING) {
            fetch(r + AHEAD * step, stage == 0 ? AHEAD : stage - 1);
            stage = stage == AHEAD ? 0 : stage + 1;
        }
        if (r + step < p.rows) {
            rstd = p.rstd[r + step];
            if constexpr (!KEPT) mean = p.mean[r + step];
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!some(k)) continue;
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const float2 d = make_float2(g[k][i], g[k][i + 1]);           // zeros past the row's end
                float2 un = make_float2(u[k][i], u[k][i + 1]);
                if constexpr (!KEPT) un = mul2(add2(un, both(-shift)), both(by));
                const float2 a = fma2(d, un, make_float2(dw[k][i], dw[k][i + 1])), c = add2(d, make_float2(db[k][i], db[k][i + 1]));
                const float2 v = mul2(d, make_float2(w[k][i], w[k][i + 1]));
                dw[k][i] = a.x, dw[k][i + 1] = a.y, db[k][i] = c.x, db[k][i + 1] = c.y;
                g[k][i] = v.x, g[k][i + 1] = v.y, u[k][i] = un.x, u[k][i + 1] = un.y;
                s1 = add2(s1, v);
                s2 = fma2(v, un, s2);
            }
        }
        float2 s = make_float2(s1.x + s1.y, s2.x + s2.y);
#pragma unroll
        for (int d = 16; d > 0; d /= 2) {
            s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, d);
            s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, d);
        }
        if constexpr (WARPS > 1) {
            if (threadIdx.x % 32 == 0) slots[group][turn][at / 32] = s;
            group_barrier<GROUP>(group);
            s = both(0.0f);
#pragma unroll
            for (int i = 0; i < WARPS; ++i) s = add2(s, slots[group][turn][i]);
            turn ^= 1;
        }
        const float a = -s.x * per_col * by, c = -s.y * per_col * by;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!some(k)) continue;
            float y[V];
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const float2 v = fma2(make_float2(g[k][i], g[k][i + 1]), both(by), fma2(make_float2(u[k][i], u[k][i + 1]), both(c), both(a)));
                y[i] = v.x, y[i + 1] = v.y;
            }
            store_row<T, WIDE>(static_cast<T *>(p.out) + r * p.out_stride, column<GROUP, NV, V>(at, k), cols, y);
        }
    }
    if (p.dweight == nullptr && p.dbias == nullptr) return;
    constexpr int N = GROUP * NV * V;
    float *const joined = reinterpret_cast<float *>(ring);      // [GROUPS][2][N]
    wait_copies<0>();
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            float4 *const to = reinterpret_cast<float4 *>(joined + group * 2 * N + column<GROUP, NV, V>(at, k) + i);
            to[0] = make_float4(dw[k][i], dw[k][i + 1], dw[k][i + 2], dw[k][i + 3]);
            to[N / 4] = make_float4(db[k][i], db[k][i + 1], db[k][i + 2], db[k][i + 3]);
        }
    __syncthreads();
    float *const part = p.joint ? joined : p.parts + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
    const int half = p.joint ? N : cols;
    for (int c = threadIdx.x; c < cols; c += THREADS) {
        float w = 0.0f, b = 0.0f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) w += joined[g * 2 * N + c], b += joined[g * 2 * N + N + c];
        part[c] = w, part[half + c] = b;
    }
    if (!p.joint) return;
    // few rows: the CTAs are a cluster, and each takes its share of the columns from all of them
    cluster_sync();
    const unsigned ctas = gridDim.x, at_all = static_cast<unsigned>(__cvta_generic_to_shared(joined));
    for (int c = blockIdx.x * THREADS + threadIdx.x; c < cols; c += ctas * THREADS) {
        float w = 0.0f, b = 0.0f;
        for (unsigned r = 0; r < ctas; ++r) w += of_cta(at_all + c * 4, r), b += of_cta(at_all + (N + c) * 4, r);
        store_param(p.dweight, p.param_bf16, c, w);
        store_param(p.dbias, p.param_bf16, c, b);
    }
    cluster_sync();                              // until all have read
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
        const float mean = cta_sum(s, slots, turn).x / static_cast<float>(p.cols);
        s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += blockDim.x) {
            const float d = Elems<T>::up(row[c]) - mean;
            s.x += d * d;
        }
        const float rstd = __frsqrt_rn(cta_sum(s, slots, turn).x / static_cast<float>(p.cols) + p.eps);
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
                encode<4>(u, true, &codes, &scale);
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
        s = cta_sum(s, slots, turn);
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
// be written over dout.  Summed in blocks of ANY_BLOCK rows, whose sums are added: taken row after row, the error would
// grow with the rows.  Ranges of 128 rows at least keep the partial sums small beside what is read, 16 ranges at least
// the device busy.  All of the backward pass from x, and from a checkpoint, in us: 4096 x 16384 bf16 458 and 347 (16 ranges
// row after row 432 and 346, ranges of 256 rows 455 and 416), 4096 x 12288 340 and 280 (343 and 280), 30000 x 8200 1536 and 1237
// (1680 and 1455).  Bound by the number of loads: element by element, and what dx needs is read again twice.
constexpr int64_t ANY_BLOCK = 64, ANY_RANGE = 128, ANY_LEAST = 16;
int64_t any_parts(int64_t rows) {
    const int64_t need = (rows + ANY_RANGE - 1) / ANY_RANGE, parts = need < ANY_LEAST ? ANY_LEAST : need < SMS ? need : SMS;
    return rows < parts ? rows : parts;
}
template <typename T, bool KEPT>
__global__ void k_norm_columns(const NormParams p) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (c >= p.cols) return;
    const int64_t lo = p.rows * blockIdx.y / gridDim.y, hi = p.rows * (blockIdx.y + 1) / gridDim.y;
    float dw = 0.0f, db = 0.0f;
    for (int64_t r = lo; r < hi; r += ANY_BLOCK) {
        const int n = static_cast<int>(hi - r < ANY_BLOCK ? hi - r : ANY_BLOCK);
        float w = 0.0f, b = 0.0f;
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float d = Elems<T>::up(static_cast<const T *>(p.dout)[(r + i) * p.dout_stride + c]);
            w += d * unit_at<T, KEPT>(p, r + i, c, mean_at<KEPT>(p, r + i), p.rstd[r + i]);
            b += d;
        }
        dw += w, db += b;
    }
    float *part = p.parts + static_cast<int64_t>(blockIdx.y) * 2 * p.cols;
    part[c] = dw;
    part[p.cols + c] = db;
}

// Sums of the partial rows: 32 columns to a CTA, 32 threads down each with four sums, then a tree;
// blockIdx.y 0 writes dweight, 1 dbias.  Rounded once, to the parameters' type.  Bound by latency (the partial rows are in
// L2): its blocks come up while k_norm_backward ends.
__global__ void __launch_bounds__(1024) k_norm_params(const NormParams p) {
    __shared__ float sums[32][33];
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x;
    void *out = blockIdx.y == 0 ? p.dweight : p.dbias;
    after_previous();
    if (out == nullptr) return;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < p.cols) {
        const float *at = p.parts + blockIdx.y * p.cols + c;
        int q = threadIdx.y;
        for (; q + 96 < p.n_parts; q += 128)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += at[static_cast<int64_t>(q + 32 * i) * 2 * p.cols];
        for (int i = 0; q < p.n_parts; q += 32, ++i) s[i] += at[static_cast<int64_t>(q) * 2 * p.cols];
    }
    sums[threadIdx.y][threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    float v = sums[threadIdx.x][threadIdx.y];          // a warp to a column
#pragma unroll
    for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int64_t to = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.y;
    if (threadIdx.x == 0 && to < p.cols) store_param(out, p.param_bf16, to, v);
}

// ------------------------------------------------------------- activations and checkpoints
// Work is laid out in vectors over rows padded to whole blocks, so that the lanes that hold a block
// are neighbours; every thread takes U vectors, a CTA's width apart, and loads all of them before it
// works on the first.
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
    unsigned vectors;                     // rows * per_row, below 2^31
    unsigned per_row, magic, shift;       // vectors to a padded row; i / per_row = (umulhi(i, magic) + i) >> shift
    int param_bf16;
};

// How a matrix is gone through: by elements, by 16-byte vectors of its rows, or, where rows follow one
// another without a gap and are made of whole blocks, as one long row (which saves the division and most
// of the address arithmetic: 116 instead of 124 us for GELU's backward pass on 16384 x 8192 bf16).
enum Mode { ELEMENTS, VECTORS, FLAT };

// A thread's vectors: their rows and columns; past the last one, a column past the row.
template <int V, int MODE>
struct Place {
    int64_t row, col;
    __device__ Place(const ElemParams &p, int u) {
        const unsigned i = blockIdx.x * (U * THREADS) + u * THREADS + threadIdx.x;
        if constexpr (MODE == FLAT) {
            row = 0;
            col = static_cast<int64_t>(i) * V;
        } else {
            const unsigned r = (__umulhi(i, p.magic) + i) >> p.shift;
            row = r;
            col = i < p.vectors ? static_cast<int64_t>(i - r * p.per_row) * V : static_cast<int64_t>(p.per_row) * V;
        }
    }
};

// GELU goes by the normal tail at a = |x|, T = 1 - Phi(a) = e q with e = exp(-a^2 / 2): it is max(x, 0) - a T, and its slope the
// step at 0 plus or minus (a phi(a) - T).  a stops at 64, where e is 0, so that an infinity meets no 0 * inf.
__device__ __forceinline__ float2 magnitude(float2 x) { return make_float2(min_nan(fabsf(x.x), 64.0f), min_nan(fabsf(x.y), 64.0f)); }

// bf16 rows: Abramowitz and Stegun, formula 7.1.26 (absolute error of erf below 1.5e-7; its coefficients halved).
__device__ __forceinline__ void normal_tail(float2 a, float2 *q, float2 *e) {
    const float2 den = fma2(a, both(0.3275911f * 0.70710678118654752f), both(1.0f));
    const float2 t = make_float2(inverse_fast(den.x), inverse_fast(den.y));
    float2 s = fma2(t, both(0.5f * 1.061405429f), both(0.5f * -1.453152027f));
    s = fma2(t, s, both(0.5f * 1.421413741f));
    s = fma2(t, s, both(0.5f * -0.284496736f));
    s = fma2(t, s, both(0.5f * 0.254829592f));
    *q = mul2(t, s);
    const float2 z = mul2(mul2(a, a), both(-0.72134752044448170f));       // - log2(e) / 2
    *e = make_float2(exp2_fast(z.x), exp2_fast(z.y));
}

// fp32 rows: T to fp32 relative to itself, and for the slope Phi around 1/2 where x is below 1.  Both polynomials are
// least-squares fits in 64 bits, weighted again and again (Lawson) until the largest relative error is least: q = t P(t) with
// t = 1 / (1 + 0.35 a) on 0 ... 14, where e underflows, to 3.2e-8; (Phi(x) - 1/2) / x in x^2 on 0 ... 1 to 7e-10.
// Error over rows of spread 1.5 in the 2-norm: 2.7e-8, of the slope 3.8e-8; with the formula above 6.9e-8 and 9.0e-8, and of a
// single value at x = -3 5e-5, now below 1e-6.  Aligned rows are bound by memory either way (16384 x 8192: 162 us, 183 with
// checkpoint, backward 237 and 184 from the checkpoint, before 180); at odd widths the arithmetic shows (16384 x 8191: 220, 221, 299
// and 263 us; 199, 211, 259 and 237 with the formula above).
__device__ __forceinline__ void normal_tail_fp32(float2 a, float2 *q, float2 *e) {
    const float2 den = fma2(a, both(0.35f), both(1.0f));
    const float2 t = make_float2(inverse_fast(den.x), inverse_fast(den.y));
    float2 s = fma2(t, both(-0.0291459185f), both(0.143971641f));
    s = fma2(t, s, both(-0.255714136f));
    s = fma2(t, s, both(0.159174027f));
    s = fma2(t, s, both(-0.0231097444f));
    s = fma2(t, s, both(0.105507966f));
    s = fma2(t, s, both(0.119832877f));
    s = fma2(t, s, both(0.139861868f));
    s = fma2(t, s, both(0.139621404f));
    *q = mul2(t, s);
    const float2 z = mul2(mul2(a, a), both(-0.72134752044448170f));
    *e = make_float2(exp2_fast(z.x), exp2_fast(z.y));
}
__device__ __forceinline__ float2 normal_near_zero(float2 x) {
    const float2 y = mul2(x, x);
    float2 s = fma2(y, both(-7.65421273e-06f), both(1.13486384e-04f));
    s = fma2(y, s, both(-1.18632995e-03f));
    s = fma2(y, s, both(9.97332342e-03f));
    s = fma2(y, s, both(-6.64903599e-02f));
    s = fma2(y, s, both(0.39894228f));
    return fma2(x, s, both(0.5f));
}
__device__ __forceinline__ float2 near_or_far(float2 a, float2 near, float2 far) { return make_float2(a.x < 1.0f ? near.x : far.x, a.y < 1.0f ? near.y : far.y); }

__device__ __forceinline__ float2 sigmoid(float2 x) {
    const float2 z = mul2(x, both(-1.4426950408889634f));
    const float2 d = add2(make_float2(exp2_fast(z.x), exp2_fast(z.y)), both(1.0f));
    return make_float2(inverse_fast(d.x), inverse_fast(d.y));
}

template <int KIND, typename T>
__device__ __forceinline__ float2 act(float2 x) {
    if constexpr (KIND == KT_GELU && sizeof(T) == 2) {
        float2 q, e;
        const float2 a = magnitude(x);
        normal_tail(a, &q, &e);
        const float2 below = mul2(mul2(q, e), make_float2(-a.x, -a.y));
        return add2(below, make_float2(max_nan(x.x, 0.0f), max_nan(x.y, 0.0f)));
    } else if constexpr (KIND == KT_GELU) {
        float2 q, e;
        const float2 a = magnitude(x);
        normal_tail_fp32(a, &q, &e);
        return fma2(mul2(q, e), make_float2(-a.x, -a.y), make_float2(max_nan(x.x, 0.0f), max_nan(x.y, 0.0f)));
    } else {
        return mul2(x, sigmoid(x));
    }
}

template <int KIND, typename T>
__device__ __forceinline__ float2 slope(float2 x) {
    if constexpr (KIND == KT_GELU && sizeof(T) == 2) {
        float2 q, e;
        const float2 a = magnitude(x);
        normal_tail(a, &q, &e);
        const float2 v = fma2(e, fma2(a, both(0.39894228040143268f), make_float2(-q.x, -q.y)), both(0.5f));
        return add2(make_float2(copysignf(v.x, x.x), copysignf(v.y, x.y)), both(0.5f));
    } else if constexpr (KIND == KT_GELU) {
        float2 q, e;
        const float2 a = magnitude(x);
        normal_tail_fp32(a, &q, &e);
        const float2 tail = mul2(q, e), far = make_float2(x.x > 0.0f ? 1.0f - tail.x : tail.x, x.y > 0.0f ? 1.0f - tail.y : tail.y);
        return fma2(make_float2(copysignf(a.x, x.x), copysignf(a.y, x.y)), mul2(e, both(0.39894228040143268f)), near_or_far(a, normal_near_zero(x), far));
    } else {
        const float2 s = sigmoid(x);
        return mul2(s, fma2(x, add2(both(1.0f), make_float2(-s.x, -s.y)), both(1.0f)));
    }
}

// The kernels on elements: U vectors to a thread, all loads before the first use, no shared memory; sixteen lanes (a warp,
// fp32) hold a checkpoint's block, whose largest magnitude goes through shuffles.  Bound by memory, on 16384 x 8192 bf16: GELU
// with checkpoint 120 us, its backward pass from the checkpoint 118 us (5715 GB/s), restore 68 us (5980 GB/s).
// At odd addresses and widths shuffles and word accesses bound them: SiLU's backward pass on 16384 x 8191 bf16 takes 221 us.
enum { KIND_NONE = -1 };                  // a checkpoint alone

template <typename T, int MODE, int KIND, bool KEEP>
__global__ void __launch_bounds__(THREADS) k_act_forward(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        raw[u] = load_row<T, MODE != ELEMENTS>(static_cast<const T *>(p.in) + at.row * p.in_stride, at.col, p.cols);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        float x[V];
        Elems<T>::widen(raw[u], x);
        if constexpr (KIND != KIND_NONE) {
            float y[V];
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const float2 v = act<KIND, T>(make_float2(x[j], x[j + 1]));
                y[j] = v.x, y[j + 1] = v.y;
            }
            store_row<T, MODE != ELEMENTS>(static_cast<T *>(p.out) + at.row * p.out_stride, at.col, p.cols, y);
        }
        if constexpr (KEEP) {
            uint2 c;
            float scale;
            encode<V>(x, true, &c, &scale);
            if (at.col < pitch_of(p.cols)) store_codes<V>(p.codes + at.row * pitch_of(p.cols) + at.col, c);
            if (at.col % BLOCK == 0 && at.col < p.cols) p.scales[at.row * blocks_of(p.cols) + at.col / BLOCK] = scale;
        }
    }
}

template <typename T, int MODE, int KIND, bool KEPT>
__global__ void __launch_bounds__(THREADS) k_act_backward(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    uint4 raw[U], raw_x[KEPT ? 1 : U];
    uint2 codes[KEPT ? U : 1];
    float scale[KEPT ? U : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        raw[u] = load_row<T, MODE != ELEMENTS>(static_cast<const T *>(p.in) + at.row * p.in_stride, at.col, p.cols);
        if constexpr (KEPT) {
            codes[u] = make_uint2(0, 0);
            scale[u] = 0.0f;
            if (at.col < p.cols) {
                codes[u] = load_codes<V>(p.codes + at.row * pitch_of(p.cols) + at.col);
                scale[u] = p.scales[at.row * blocks_of(p.cols) + at.col / BLOCK];
            }
        } else {
            raw_x[u] = load_row<T, MODE != ELEMENTS>(static_cast<const T *>(p.x) + at.row * p.x_stride, at.col, p.cols);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        float d[V], x[V];
        Elems<T>::widen(raw[u], d);
        if constexpr (KEPT) decode<V>(codes[u], scale[u], x);
        else Elems<T>::widen(raw_x[u], x);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 v = mul2(make_float2(d[j], d[j + 1]), slope<KIND, T>(make_float2(x[j], x[j + 1])));
            d[j] = v.x, d[j + 1] = v.y;
        }
        store_row<T, MODE != ELEMENTS>(static_cast<T *>(p.out) + at.row * p.out_stride, at.col, p.cols, d);
    }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(THREADS) k_restore(const ElemParams p) {
    constexpr int V = Elems<T>::V;
    uint2 codes[U];
    float scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        codes[u] = make_uint2(0, 0);
        scale[u] = 0.0f;
        if (at.col < p.cols) {
            codes[u] = load_codes<V>(p.codes + at.row * pitch_of(p.cols) + at.col);
            scale[u] = p.scales[at.row * blocks_of(p.cols) + at.col / BLOCK];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place<V, MODE> at(p, u);
        float x[V];
        decode<V>(codes[u], scale[u], x);
        if ((p.weight != nullptr || p.bias != nullptr) && at.col < p.cols) {
            float w[V], b[V];
            load_param(p.weight, p.param_bf16, at.col, p.cols, 1.0f, w);
            load_param(p.bias, p.param_bf16, at.col, p.cols, 0.0f, b);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = x[j] * w[j] + b[j];
        }
        store_row<T, MODE != ELEMENTS>(static_cast<T *>(p.out) + at.row * p.out_stride, at.col, p.cols, x);
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

int check_per_row(const float *mean, const float *rstd) {
    for (const float *p : {mean, rstd})
        if (reinterpret_cast<uintptr_t>(p) % 4) return fail(KT_ERR_ALIGN, "mean or rstd is not 4-byte aligned");
    return KT_OK;
}

// 128-bit accesses: base and row stride multiples of 16 bytes, whole vectors in a row.
bool wide(const void *p, int64_t stride, int64_t rows, int64_t cols, int dtype) {
    const int64_t es = elem_size(dtype);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols * es % 16 == 0 && (rows <= 1 || stride * es % 16 == 0);
}

// How many threads share a row: a warp where it can hold the row, else a CTA of up to 512.
struct RowShape {
    int group, nv, threads;
};
// The least that holds the row: what a row takes hardly depends on how many of its threads have columns (16384 rows bf16, with
// 128, 256 or 512 threads only and now, in us: forward on 2560 columns 50 and 35, on 5120 columns 123 and 74; backward from a
// checkpoint on 2560 columns 63 and 49, on 640 columns 25 and 20).
constexpr int GROUPS_OF_ROW[] = {64, 96, 128, 160, 192, 256, 320, 384, 512};
RowShape row_shape(int64_t cols, int dtype) {
    const int v = dtype == KT_F32 ? 4 : 8;
    const int64_t vectors = (pitch_of(cols) + v - 1) / v;
    RowShape s{};
    s.group = 32;
    if (vectors > 32 * (E / v))
        for (int group : GROUPS_OF_ROW)
            if (vectors <= static_cast<int64_t>(s.group = group) * (E / v)) break;
    s.threads = s.group == 32 ? 128 : s.group;
    s.nv = s.group == 32 ? static_cast<int>((vectors + 31) / 32) : E / v;
    if (s.nv == 3) s.nv = 4;
    return s;
}

// (A kernel's limit of shared memory is raised once per device: the call costs a third of a launch.)
template <auto KERNEL>
int start_norm_kernel(const NormParams &p, int grid, int threads, size_t smem, cudaStream_t st) {
    static std::atomic<uint64_t> raised{0};
    int dev = 0;
    KT_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (smem > 47 * 1024 && (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit))) {
        KT_CUDA(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        raised.fetch_or(bit, std::memory_order_relaxed);
    }
    if (p.joint) {
        KT_CUDA(launch_joint(KERNEL, grid, dim3(grid), dim3(threads), smem, st, p));
        return KT_OK;
    }
    KERNEL<<<grid, threads, smem, st>>>(p);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

template <typename T, bool WIDE, int GROUP, int NV>
int start_norm(bool backward, const NormParams &p, int grid, cudaStream_t st) {
    constexpr int V = Elems<T>::V, FORWARD = norm_threads<GROUP>(), WARP = in_ring<T, WIDE>() ? (rows_ahead<NV>() + 1) * NV * cells_of_warp<WIDE>() : 0;      // a warp's cells
    if (!backward) return start_norm_kernel<k_norm_forward<T, WIDE, GROUP, NV>>(p, grid, FORWARD, WARP * FORWARD / 32 * sizeof(uint4), st);
    constexpr int BACKWARD = backward_threads<GROUP>();
    const size_t joined = 2 * BACKWARD * NV * V * sizeof(float);
    const size_t kept = WARP * BACKWARD / 32 * (sizeof(uint4) + V + sizeof(float)), whole = WARP * BACKWARD / 32 * 2 * sizeof(uint4);
    if (p.codes != nullptr) return start_norm_kernel<k_norm_backward<T, WIDE, GROUP, NV, true>>(p, grid, BACKWARD, kept > joined ? kept : joined, st);
    return start_norm_kernel<k_norm_backward<T, WIDE, GROUP, NV, false>>(p, grid, BACKWARD, whole > joined ? whole : joined, st);
}

template <typename T, bool WIDE>
int start_norm(bool backward, const RowShape &s, const NormParams &p, int grid, cudaStream_t st) {
    constexpr int MOST = E / Elems<T>::V;
    switch (s.group) {
        case 32:
            if (s.nv == 1) return start_norm<T, WIDE, 32, 1>(backward, p, grid, st);
            if (s.nv == 2) return start_norm<T, WIDE, 32, 2>(backward, p, grid, st);
            return start_norm<T, WIDE, 32, MOST>(backward, p, grid, st);
        case 64: return start_norm<T, WIDE, 64, MOST>(backward, p, grid, st);
        case 96: return start_norm<T, WIDE, 96, MOST>(backward, p, grid, st);
        case 128: return start_norm<T, WIDE, 128, MOST>(backward, p, grid, st);
        case 160: return start_norm<T, WIDE, 160, MOST>(backward, p, grid, st);
        case 192: return start_norm<T, WIDE, 192, MOST>(backward, p, grid, st);
        case 256: return start_norm<T, WIDE, 256, MOST>(backward, p, grid, st);
        case 320: return start_norm<T, WIDE, 320, MOST>(backward, p, grid, st);
        case 384: return start_norm<T, WIDE, 384, MOST>(backward, p, grid, st);
        default: return start_norm<T, WIDE, 512, MOST>(backward, p, grid, st);
    }
}

int start_norm(bool backward, int dtype, bool wide_, const RowShape &s, const NormParams &p, int grid, cudaStream_t st) {
    if (dtype == KT_F32) return wide_ ? start_norm<float, true>(backward, s, p, grid, st) : start_norm<float, false>(backward, s, p, grid, st);
    return wide_ ? start_norm<__nv_bfloat16, true>(backward, s, p, grid, st) : start_norm<__nv_bfloat16, false>(backward, s, p, grid, st);
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

// Runs start(p, mode, ctas) over the rows, in pieces of fewer than 2^30 vectors.  `wide`: all matrices allow 128-bit accesses.
template <typename Start>
int over_rows(ElemParams p, int dtype, bool wide_, Start start) {
    const int v = dtype == KT_F32 ? 4 : 8, es = elem_size(dtype);
    int mode = wide_ ? VECTORS : ELEMENTS;
    const bool gapless = p.rows == 1 || ((!p.in || p.in_stride == p.cols) && (!p.x || p.x_stride == p.cols) && (!p.out || p.out_stride == p.cols));
    if (wide_ && gapless && p.cols % BLOCK == 0 && p.weight == nullptr && p.bias == nullptr) {
        // one row, cut into rows of 2^20 blocks at most where it is longer than that
        mode = FLAT;
        const int64_t all = p.rows * p.cols, most = static_cast<int64_t>(BLOCK) << 20;
        p.rows = 1;
        for (int64_t at = 0; at < all; at += most) {
            ElemParams q = p;
            q.cols = all - at < most ? all - at : most;
            q.vectors = static_cast<unsigned>(q.cols / v);
            auto past = [&](const void *from) { return from ? static_cast<const char *>(from) + at * es : nullptr; };
            q.in = past(p.in), q.x = past(p.x), q.out = const_cast<char *>(past(p.out));
            q.codes = p.codes ? p.codes + at : nullptr, q.scales = p.scales ? p.scales + at / BLOCK : nullptr;
            start(q, mode, static_cast<int>((q.vectors + U * THREADS - 1) / (U * THREADS)));
            KT_CUDA(cudaGetLastError());
        }
        return KT_OK;
    }
    p.per_row = static_cast<unsigned>(blocks_of(p.cols) * (BLOCK / v));
    for (p.shift = 0; (1u << p.shift) < p.per_row;) ++p.shift;
    p.magic = static_cast<unsigned>(((1ull << 32) * ((1ull << p.shift) - p.per_row)) / p.per_row + 1);
    const int64_t piece = (INT64_C(1) << 30) / p.per_row, all = p.rows;
    for (int64_t r = 0; r < all; r += piece) {
        ElemParams q = p;
        q.rows = all - r < piece ? all - r : piece;
        q.vectors = static_cast<unsigned>(q.rows * q.per_row);
        auto past = [&](const void *at, int64_t stride) { return at ? static_cast<const char *>(at) + r * stride * es : nullptr; };
        q.in = past(p.in, p.in_stride), q.x = past(p.x, p.x_stride), q.out = const_cast<char *>(past(p.out, p.out_stride));
        q.codes = p.codes ? p.codes + r * pitch_of(p.cols) : nullptr, q.scales = p.scales ? p.scales + r * blocks_of(p.cols) : nullptr;
        start(q, mode, static_cast<int>((q.vectors + U * THREADS - 1) / (U * THREADS)));
        KT_CUDA(cudaGetLastError());
    }
    return KT_OK;
}

template <typename T, int MODE>
void start_act_forward(const ElemParams &p, int kind, int ctas, cudaStream_t st) {
    const bool keep = p.codes != nullptr;
    if (kind == KT_GELU) keep ? k_act_forward<T, MODE, KT_GELU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_forward<T, MODE, KT_GELU, false><<<ctas, THREADS, 0, st>>>(p);
    else if (kind == KT_SILU) keep ? k_act_forward<T, MODE, KT_SILU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_forward<T, MODE, KT_SILU, false><<<ctas, THREADS, 0, st>>>(p);
    else k_act_forward<T, MODE, KIND_NONE, true><<<ctas, THREADS, 0, st>>>(p);
}

template <typename T, int MODE>
void start_act_backward(const ElemParams &p, int kind, int ctas, cudaStream_t st) {
    const bool kept = p.codes != nullptr;
    if (kind == KT_GELU) kept ? k_act_backward<T, MODE, KT_GELU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_backward<T, MODE, KT_GELU, false><<<ctas, THREADS, 0, st>>>(p);
    else kept ? k_act_backward<T, MODE, KT_SILU, true><<<ctas, THREADS, 0, st>>>(p) : k_act_backward<T, MODE, KT_SILU, false><<<ctas, THREADS, 0, st>>>(p);
}

template <typename T, int MODE>
void start_restore(const ElemParams &p, int, int ctas, cudaStream_t st) {
    k_restore<T, MODE><<<ctas, THREADS, 0, st>>>(p);
}

#define KT_EACH(start)                                                                                                  \
    [&](const ElemParams &p, int mode, int ctas) {                                                                      \
        if (dtype == KT_F32)                                                                                            \
            mode == FLAT ? start<float, FLAT>(p, kind, ctas, st) : mode == VECTORS ? start<float, VECTORS>(p, kind, ctas, st) : start<float, ELEMENTS>(p, kind, ctas, st); \
        else                                                                                                            \
            mode == FLAT      ? start<__nv_bfloat16, FLAT>(p, kind, ctas, st)                                           \
            : mode == VECTORS ? start<__nv_bfloat16, VECTORS>(p, kind, ctas, st)                                        \
                              : start<__nv_bfloat16, ELEMENTS>(p, kind, ctas, st);                                      \
    }
int act_forward(const ElemParams &all, int dtype, int kind, bool wide_, cudaStream_t st) { return over_rows(all, dtype, wide_, KT_EACH(start_act_forward)); }
int act_backward(const ElemParams &all, int dtype, int kind, bool wide_, cudaStream_t st) { return over_rows(all, dtype, wide_, KT_EACH(start_act_backward)); }
int restore(const ElemParams &all, int dtype, int kind, bool wide_, cudaStream_t st) { return over_rows(all, dtype, wide_, KT_EACH(start_restore)); }
#undef KT_EACH

// CTAs of the backward pass.  Up to CLUSTER of them, with up to four rows to a group, are a cluster, which saves the
// second kernel (109 rows of 512, both together: 13.1 -> 6.9 us); else there is a row of partial sums to each, and a CTA has
// eight rows at least, or two to a group, so that these stay small beside what is read (with two rows to each of eight or
// more groups: 1500 x 500 bf16 10.3 us, now 8.7; 4000 x 300 10.4, now 11.2).
constexpr int64_t CLUSTER = 8;
int64_t norm_parts(int64_t rows, const RowShape &s, bool *joint) {
    const int64_t groups = GROUP_MAX / s.group;
    const int64_t least = groups < 8 ? groups * 2 : groups;
    *joint = rows <= CLUSTER * groups * 4;
    const int64_t need = *joint ? (rows + groups - 1) / groups : (rows + least - 1) / least, most = *joint ? CLUSTER : SMS;
    return need < most ? need : most;
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
    if (int rc = check_per_row(mean, rstd)) return rc;
    NormParams p{};
    p.x = x, p.weight = weight, p.bias = bias, p.out = out, p.mean = mean, p.rstd = rstd, p.codes = codes, p.scales = scales;
    p.rows = rows, p.cols = cols, p.x_stride = x_stride, p.out_stride = out_stride, p.eps = eps, p.param_bf16 = param_dtype == KT_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cols > ROW_MAX) {
        const int grid = static_cast<int>(rows < SMS * 4 ? rows : SMS * 4);
        if (dtype == KT_F32) start_norm_any<float>(false, p, grid, st);
        else start_norm_any<__nv_bfloat16>(false, p, grid, st);
        KT_CUDA(cudaGetLastError());
        return KT_OK;
    }
    const RowShape s = row_shape(cols, dtype);
    const int per_cta = s.threads / s.group;
    const bool w = wide(x, x_stride, rows, cols, dtype) && wide(out, out_stride, rows, cols, dtype);
    const int64_t need = (rows + per_cta - 1) / per_cta, most = static_cast<int64_t>(SMS) * (forward_threads(s.nv * (dtype == KT_F32 ? 4 : 8)) / s.threads);
    return start_norm(false, dtype, w, s, p, static_cast<int>(need < most ? need : most), st);
}

int64_t kt_norm_workspace(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return 0;
    int64_t parts = any_parts(rows);
    if (cols <= ROW_MAX)                  // room for either type
        for (int dtype : {KT_F32, KT_BF16}) {
            bool joint = false;
            const int64_t n = norm_parts(rows, row_shape(cols, dtype), &joint);
            parts = dtype == KT_F32 || n > parts ? n : parts;
        }
    return parts * 2 * cols * static_cast<int64_t>(sizeof(float));
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
        if (int rc = check_per_row(mean, rstd)) return rc;
        if (sums) {
            const int64_t need = kt_norm_workspace(rows, cols);
            if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
            if (workspace_bytes < need) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)workspace_bytes, (long long)need);
            if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
        }
    }
    NormParams p{};
    p.dout = dout, p.x = x, p.weight = weight, p.out = dx, p.mean = const_cast<float *>(mean), p.rstd = const_cast<float *>(rstd);
    p.codes = const_cast<int8_t *>(codes), p.scales = const_cast<float *>(scales), p.dweight = dweight, p.dbias = dbias;
    p.parts = sums ? static_cast<float *>(workspace) : nullptr;
    p.rows = rows, p.cols = cols, p.dout_stride = dout_stride, p.x_stride = x_stride, p.out_stride = dx_stride, p.param_bf16 = param_dtype == KT_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows > 0 && cols > ROW_MAX) {
        p.n_parts = static_cast<int>(any_parts(rows));
        const int grid = static_cast<int>(rows < SMS * 4 ? rows : SMS * 4);
        if (dtype == KT_F32) start_norm_any<float>(true, p, grid, st);
        else start_norm_any<__nv_bfloat16>(true, p, grid, st);
        KT_CUDA(cudaGetLastError());
    } else if (rows > 0) {
        const RowShape s = row_shape(cols, dtype);
        const bool w = wide(dout, dout_stride, rows, cols, dtype) && wide(dx, dx_stride, rows, cols, dtype) && (x == nullptr || wide(x, x_stride, rows, cols, dtype));
        bool joint = false;
        p.n_parts = static_cast<int>(norm_parts(rows, s, &joint));
        p.joint = joint && sums;
        if (int rc = start_norm(true, dtype, w, s, p, p.n_parts, st)) return rc;
    }
    if (sums && !p.joint) {
        KT_CUDA(launch_behind(k_norm_params, 1, dim3(static_cast<unsigned>((cols + 31) / 32), 2), dim3(32, 32), 0, st, p));
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
    return act_forward(p, dtype, KIND_NONE, wide(x, x_stride, rows, cols, dtype), static_cast<cudaStream_t>(stream));
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
    return restore(p, dtype, KIND_NONE, wide(out, out_stride, rows, cols, dtype), static_cast<cudaStream_t>(stream));
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
    return act_forward(p, dtype, kind, wide(x, x_stride, rows, cols, dtype) && wide(out, out_stride, rows, cols, dtype), static_cast<cudaStream_t>(stream));
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
    const bool w = wide(dout, dout_stride, rows, cols, dtype) && wide(dx, dx_stride, rows, cols, dtype) && (x == nullptr || wide(x, x_stride, rows, cols, dtype));
    return act_backward(p, dtype, kind, w, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
