// kt_orth.cu -- a matrix-shaped update orthogonalised by Newton-Schulz products.  Contract: include/kaitian.h.
//
//   X <- G / |G|_F;  `steps` times  A = X X^T,  X <- (a I + b A + c A^2) X;  out = scale X
// with X^T in place of X where G has more rows than columns, so that A has the shorter side.  The polynomial
// a s + b s^3 + c s^5 takes every singular value s towards one.
//
// Three products a step (kt_product.cuh), in fp16 with fp32 sums: everything that is held between products has a known
// range (singular values of X at most some 1.2, of A 1.5, of the factor |a|), so that fp16's 11 bits can be had where
// bf16, whose range is not needed, has 8: the result is as far from 64 bits as one in 32 bits rounded to bf16.
// Powers of two keep small entries off fp16's subnormals: X is held times 2^7, A times 2^14, the factor times 2^13.
// A and the factor are symmetric: tiles on and above the diagonal are computed, and written to both sides.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <cmath>

#include "kt_eight.cuh"
#include "kt_internal.h"
#include "kt_pairs.cuh"
#include "kt_product.cuh"

using namespace ktd;

namespace {

constexpr float X_UNIT = 128.0f, A_UNIT = 16384.0f, FACTOR_UNIT = 8192.0f;
constexpr int SUM_BLOCKS = 256;                 // partial sums of squares to a matrix, at most: a thread reads one

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ------------------------------------------------------------------------------------ start
struct StartParams {
    const void *x;
    int64_t stride[2];                          // matrix, row
    int64_t rows, cols, pitch;                  // pitch: of X, in elements
    double *sums;
    int sum_blocks;                             // CTAs, each with a sum, to a matrix
    __half *to;
};

// Sums of squares in 64 bits: no element is too large or too small for them.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256) k_orth_squares(const StartParams p) {
    __shared__ double of_warp[8];
    let_next_begin();
    const uint32_t cols = static_cast<uint32_t>(p.cols), pieces = (cols + 7) / 8, all = static_cast<uint32_t>(p.rows) * pieces, step = gridDim.x * 256;      // 2^29 pieces at most
    const T *const x = static_cast<const T *>(p.x) + blockIdx.y * p.stride[0];
    double sum[2] = {0.0, 0.0};
    for (uint32_t i0 = blockIdx.x * 256 + threadIdx.x; i0 < all; i0 += 4 * step) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t i = i0 + u * step, r = i < all ? i / pieces : 0, c = i < all ? (i - r * pieces) * 8 : cols;      // (past the last column: zeros)
            read_eight<T, WHOLE>(x + r * p.stride[1], c, p.cols, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = v[u][e];
                sum[e % 2] = fma(d, d, sum[e % 2]);
            }
    }
    double all_of = sum[0] + sum[1];
#pragma unroll
    for (int far = 16; far; far /= 2) all_of += __shfl_xor_sync(0xFFFFFFFFu, all_of, far);
    if (threadIdx.x % 32 == 0) of_warp[threadIdx.x / 32] = all_of;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) all_of += of_warp[w];
        p.sums[blockIdx.y * gridDim.x + blockIdx.x] = all_of;
    }
}

// X = G / |G| in fp16.  A matrix of zeros stays one; one with an infinity or a NaN becomes NaN throughout.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256) k_orth_start(const StartParams p) {
    __shared__ double of_warp[8];
    let_next_begin();
    after_previous();
    const uint32_t cols = static_cast<uint32_t>(p.cols), pieces = (cols + 7) / 8, all = static_cast<uint32_t>(p.rows) * pieces, step = gridDim.x * 256;      // 2^29 pieces at most
    double sum = static_cast<int>(threadIdx.x) < p.sum_blocks ? p.sums[blockIdx.y * p.sum_blocks + threadIdx.x] : 0.0;
#pragma unroll
    for (int far = 16; far; far /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, far);
    if (threadIdx.x % 32 == 0) of_warp[threadIdx.x / 32] = sum;
    __syncthreads();
    sum = of_warp[0];
    for (int w = 1; w < 8; ++w) sum += of_warp[w];
    const double by = sum == 0.0 ? 0.0 : isfinite(sum) ? X_UNIT / sqrt(sum) : __longlong_as_double(0x7FF8000000000000ll);
    const bool narrow = by < 1e30 && by > 1e-30;       // fp32 holds the factor
    const float by32 = static_cast<float>(by);
    const T *const x = static_cast<const T *>(p.x) + blockIdx.y * p.stride[0];
    __half *const to = p.to + blockIdx.y * p.rows * p.pitch;
    for (uint32_t i0 = blockIdx.x * 256 + threadIdx.x; i0 < all; i0 += 4 * step) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t i = i0 + u * step, r = i < all ? i / pieces : 0, c = i < all ? (i - r * pieces) * 8 : cols;
            read_eight<T, WHOLE>(x + r * p.stride[1], c, p.cols, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t i = i0 + u * step, r = i / pieces, c = (i - r * pieces) * 8;
            if (i >= all) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = narrow ? v[u][e] * by32 : static_cast<float>(v[u][e] * by);
            uint4 w;
            w.x = pack_half(v[u][0], v[u][1]), w.y = pack_half(v[u][2], v[u][3]), w.z = pack_half(v[u][4], v[u][5]), w.w = pack_half(v[u][6], v[u][7]);
            *reinterpret_cast<uint4 *>(to + r * p.pitch + c) = w;
        }
    }
}

// ------------------------------------------------------------------------------------ products
struct OrthParams {
    int rows, cols, tiles_m, tiles_n, batch, steps;        // of the result; stages of the reduction
    int whole;                                  // both sides of a symmetric result are computed
    int64_t pitch;                              // of a symmetric result, in elements
    const __half *gram;                         // A, for the factor
    float a, b, c;
    void *out;                                  // of the last product
    int64_t out_stride[2];
};

// 32 values of the thread's row as fp16 into half of the store's rows.
__device__ __forceinline__ void pack_halves(const Part &part, int half, const float (&x)[32]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint4 v;
        v.x = pack_half(x[u * 8], x[u * 8 + 1]), v.y = pack_half(x[u * 8 + 2], x[u * 8 + 3]), v.z = pack_half(x[u * 8 + 4], x[u * 8 + 5]), v.w = pack_half(x[u * 8 + 6], x[u * 8 + 7]);
        *part.piece(half * 4 + u) = v;
    }
}

// A symmetric matrix: A (FACTOR false, from X along or down its rows) or the factor a I + b A + c A^2 (from A).
// The mirrored side of 32 x 32 values goes through shared memory, where lanes are columns: two lanes swap halves, so
// that each writes two neighbours of one row.  (Two-byte stores straight to memory took 27 us to a tile, more than its product.)
template <bool PAIR_, bool DOWN, bool FACTOR>
struct SymmetricTask : InTurn<SymmetricTask<PAIR_, DOWN, FACTOR>, OrthParams> {
    using Params = OrthParams;
    static constexpr bool PAIR = PAIR_, HALF = true;
    static constexpr int SIDE = PAIR ? 256 : 128;
    __device__ static int each(const Params &p) { return p.whole ? p.tiles_m * p.tiles_m : p.tiles_m * (p.tiles_m + 1) / 2; }
    __device__ static int tiles(const Params &p) { return each(p) * p.batch; }
    __device__ static bool a_down(const Tile &) { return DOWN; }
    __device__ static bool b_down(const Tile &) { return DOWN; }
    __device__ static const CUtensorMap *map_a(const ProductMaps &maps, const Params &, const Tile &) { return &maps.a; }
    __device__ static const CUtensorMap *map_b(const ProductMaps &maps, const Params &, const Tile &) { return &maps.b; }
    __device__ static Tile tile_at(const Params &p, int i) {
        const int z = i / each(p);
        int m = 0, n = i - z * each(p);
        if (p.whole) return {n / p.tiles_m * SIDE, n % p.tiles_m * SIDE, z, 0, p.steps, 0, 0};
        for (; n >= p.tiles_m - m; ++m) n -= p.tiles_m - m;
        return {m * SIDE, (m + n) * SIDE, z, 0, p.steps, 0, 0};
    }
    __device__ static void finish(const Params &p, const ProductMaps &maps, const Tile &t, Part &part) {
        if (part.warp_row >= p.rows) return;
        const int lane = threadIdx.x % 32;
        const bool mirrored = !p.whole && t.n != t.m;
        uint4 g[4] = {};
        auto of_gram = [&](int c0) {            // (rows of A are whole vectors, whatever lies past their last element)
            if (!FACTOR || part.row >= p.rows || c0 >= p.rows) return;
            const uint4 *from = reinterpret_cast<const uint4 *>(p.gram + (static_cast<int64_t>(t.z) * p.rows + part.row) * p.pitch + c0);
#pragma unroll
            for (int u = 0; u < 4; ++u) g[u] = from[u];
        };
        of_gram(part.col);
        over_columns<SIDE / 2>(part, [&](int c0, auto half, uint32_t (&r)[32]) {
            if (c0 >= p.rows) return;
            uint32_t v[16];
            [[maybe_unused]] const int d = part.row - c0;
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                float2 x = pair_of(r, e);
                if constexpr (FACTOR) {
                    const uint32_t w = e % 8 / 2 == 0 ? g[e / 8].x : e % 8 / 2 == 1 ? g[e / 8].y : e % 8 / 2 == 2 ? g[e / 8].z : g[e / 8].w;
                    const float2 in = __half22float2(*reinterpret_cast<const __half2 *>(&w));
                    x = fma2(in, both(p.b * (FACTOR_UNIT / A_UNIT)), mul2(x, both(p.c * (FACTOR_UNIT / A_UNIT / A_UNIT))));
                    if (e == d) x.x += p.a * FACTOR_UNIT;
                    if (e + 1 == d) x.y += p.a * FACTOR_UNIT;
                }
                v[e / 2] = pack_half(x.x, x.y);
            }
            of_gram(c0 + 32);
            part.store_next();
#pragma unroll
            for (int u = 0; u < 4; ++u)         // rows of 64 bytes, in the 64-byte swizzle
                *reinterpret_cast<uint4 *>(part.store + lane * 64 + ((u ^ (lane / 2 & 3)) << 4)) = make_uint4(v[u * 4], v[u * 4 + 1], v[u * 4 + 2], v[u * 4 + 3]);
            if (mirrored) {
                uint8_t *const mirror = part.store + STORE_BYTES / 2 + (lane & 1) * 64 + (lane & ~1) * 2;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t theirs = __shfl_xor_sync(0xFFFFFFFFu, v[e], 1);
                    *reinterpret_cast<uint32_t *>(mirror + e * 128) = lane & 1 ? (theirs >> 16) | (v[e] & 0xFFFF0000u) : (v[e] & 0xFFFFu) | (theirs << 16);
                }
            }
            part.send(&maps.out, c0, part.warp_row, t.z, false, mirrored ? &maps.out2 : nullptr, STORE_BYTES / 2, part.warp_row, c0);
        });
    }
};

// The next X: factor times X (WIDE), or X times factor; the last time to the result.
template <bool PAIR_, bool WIDE, bool LAST>
struct ApplyTask : InTurn<ApplyTask<PAIR_, WIDE, LAST>, OrthParams> {
    using Params = OrthParams;
    static constexpr bool PAIR = PAIR_, HALF = true;
    static constexpr int SIDE = PAIR ? 256 : 128;
    __device__ static int tiles(const Params &p) { return p.tiles_m * p.tiles_n * p.batch; }
    __device__ static bool a_down(const Tile &) { return false; }
    __device__ static bool b_down(const Tile &) { return WIDE; }
    __device__ static const CUtensorMap *map_a(const ProductMaps &maps, const Params &, const Tile &) { return &maps.a; }
    __device__ static const CUtensorMap *map_b(const ProductMaps &maps, const Params &, const Tile &) { return &maps.b; }
    __device__ static Tile tile_at(const Params &p, int i) {
        const int each = p.tiles_m * p.tiles_n, z = i / each, in = i - z * each, band = in / (8 * p.tiles_n), left = in - band * 8 * p.tiles_n, high = min(8, p.tiles_m - band * 8);
        return {(band * 8 + left % high) * SIDE, left / high * SIDE, z, 0, p.steps, 0, 0};
    }
    __device__ static void finish(const Params &p, const ProductMaps &maps, const Tile &t, Part &part) {
        if (part.warp_row >= p.rows) return;
        over_columns<SIDE / 2>(part, [&](int c0, auto half, uint32_t (&r)[32]) {
            if (c0 - half * 32 >= p.cols) return;
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(r[e]) * p.a;
            if constexpr (!LAST) {
                if (half == 0) part.store_next();
                pack_halves(part, half, x);
                if (half == 1) part.send(&maps.out, c0 - 32, part.warp_row, t.z);
            } else if (part.row < p.rows && c0 < p.cols) {
                __nv_bfloat16 *const row = static_cast<__nv_bfloat16 *>(p.out) + t.z * p.out_stride[0] + part.row * p.out_stride[1] + c0;
                if (c0 + 32 <= p.cols && reinterpret_cast<uintptr_t>(row) % 16 == 0) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 v;
                        v.x = pack_bf16(x[e], x[e + 1]), v.y = pack_bf16(x[e + 2], x[e + 3]), v.z = pack_bf16(x[e + 4], x[e + 5]), v.w = pack_bf16(x[e + 6], x[e + 7]);
                        *reinterpret_cast<uint4 *>(row + e) = v;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c0 + e < p.cols) row[e] = __float2bfloat16_rn(x[e]);
                }
            }
        });
    }
};

// ---------------------------------------------------------------------------------- host side
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct Plan {
    int64_t batch, rows, cols, side, pitch_x, pitch_a;
    bool wide;
    int64_t at_x[2], at_gram, at_factor, bytes;           // the sums of squares come first
    Plan(int64_t b, int64_t r, int64_t c) : batch(b), rows(r), cols(c), side(r < c ? r : c), pitch_x(up(c, 64)), pitch_a(up(side, 64)), wide(r <= c) {
        int64_t at = up(batch * SUM_BLOCKS * 8, 1024);
        for (int64_t &x : at_x) x = at, at += up(batch * rows * pitch_x * 2, 1024);
        at_gram = at, at += up(batch * side * pitch_a * 2, 1024);
        at_factor = at, at += up(batch * side * pitch_a * 2, 1024);
        bytes = at;
    }
};

// The largest singular value that each step can meet, from one on (|G|_F bounds it), tells whether fp16 holds all
// that is kept between products.
int check_polynomial(int steps, float a, float b, float c) {
    double most = 1.0;
    for (int i = 0; i < steps; ++i) {
        double next = 0.0, factor = 0.0;
        for (int j = 0; j <= 512; ++j) {
            const double s = most * j / 512, f = a + s * s * (b + s * s * c);
            next = std::fmax(next, std::fabs(s * f)), factor = std::fmax(factor, std::fabs(f));
        }
        // (a sample in 512 is within 1 % of the largest value of a polynomial of such degree and size; roundings add less)
        if (!(factor <= 7.5) || !(next <= 1.9)) return fail(KT_ERR_INVALID, "these coefficients take singular values to %.3g in step %d: up to 1.9 is held", next, i + 1);
        most = next * 1.01;
    }
    return KT_OK;
}

int64_t tiles_of(int64_t x, int side) { return (x + side - 1) / side; }

template <bool PAIR>
int run(const Plan &plan, char *ws, int steps, float a, float b, float c, float scale, void *out, const int64_t *out_stride, cudaStream_t st) {
    constexpr int SIDE = PAIR ? 256 : 128;
    const int64_t matrix_x = plan.rows * plan.pitch_x * 2, matrix_a = plan.side * plan.pitch_a * 2, symmetric = tiles_of(plan.side, SIDE);
    char *const gram = ws + plan.at_gram, *const factor = ws + plan.at_factor;
    ProductMaps g{}, f{}, x{};
    const CUtensorMapDataType half = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    for (int i = 0; i < 4; ++i)       // what both write, and its mirrored side
        if (int rc = describe_matrix(i == 0 ? &g.out : i == 1 ? &g.out2 : i == 2 ? &f.out : &f.out2, "the workspace", half, 2, i < 2 ? gram : factor, plan.side, plan.side, plan.batch, plan.pitch_a * 2,
                                     matrix_a, 32, 32, i % 2 == 0))
            return rc;
    if (int rc = describe_operand(&f.a, "the workspace", true, false, gram, plan.side, plan.side, plan.batch, plan.pitch_a * 2, matrix_a)) return rc;
    f.b = f.a;
    CUtensorMap of_factor;
    if (int rc = describe_operand(&of_factor, "the workspace", true, false, factor, plan.side, plan.side, plan.batch, plan.pitch_a * 2, matrix_a)) return rc;
    OrthParams pg{};
    pg.rows = pg.cols = static_cast<int>(plan.side), pg.tiles_m = pg.tiles_n = static_cast<int>(symmetric), pg.batch = static_cast<int>(plan.batch), pg.pitch = plan.pitch_a;
    // Where every tile of the whole square gets a worker of its own, mirroring would only make each take longer.
    pg.whole = symmetric * symmetric * plan.batch <= PRODUCT_SMS / (PAIR ? 2 : 1);
    OrthParams pf = pg, px{};
    pg.steps = static_cast<int>(tiles_of(plan.wide ? plan.cols : plan.rows, K_STEP));
    pf.steps = static_cast<int>(tiles_of(plan.side, K_STEP)), pf.gram = reinterpret_cast<const __half *>(gram);
    pf.a = a, pf.b = b, pf.c = c;
    px.rows = static_cast<int>(plan.rows), px.cols = static_cast<int>(plan.cols), px.tiles_m = static_cast<int>(tiles_of(plan.rows, SIDE)), px.tiles_n = static_cast<int>(tiles_of(plan.cols, SIDE));
    px.batch = pg.batch, px.steps = pf.steps, px.out = out, px.out_stride[0] = out_stride[0], px.out_stride[1] = out_stride[1];
    const int64_t tiles_a = (pg.whole ? symmetric * symmetric : symmetric * (symmetric + 1) / 2) * plan.batch, tiles_x = static_cast<int64_t>(px.tiles_m) * px.tiles_n * plan.batch;
    for (int i = 0; i < steps; ++i) {
        char *const now = ws + plan.at_x[i % 2], *const next = ws + plan.at_x[(i + 1) % 2];
        const bool last = i + 1 == steps;
        if (int rc = describe_operand(&g.a, "the workspace", true, !plan.wide, now, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x)) return rc;
        g.b = g.a;
        if (int rc = plan.wide ? start_product<SymmetricTask<PAIR, false, false>>(g, pg, tiles_a, st) : start_product<SymmetricTask<PAIR, true, false>>(g, pg, tiles_a, st)) return rc;
        if (int rc = start_product<SymmetricTask<PAIR, false, true>>(f, pf, tiles_a, st)) return rc;
        CUtensorMap of_x;
        if (int rc = describe_operand(&of_x, "the workspace", true, plan.wide, now, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x)) return rc;
        x.a = plan.wide ? of_factor : of_x, x.b = plan.wide ? of_x : of_factor;
        if (int rc = describe_matrix(&x.out, "the workspace", half, 2, next, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x, 64, 32)) return rc;
        px.a = last ? scale / (FACTOR_UNIT * X_UNIT) : 1.0f / FACTOR_UNIT;
        int rc;
        if (plan.wide) rc = last ? start_product<ApplyTask<PAIR, true, true>>(x, px, tiles_x, st) : start_product<ApplyTask<PAIR, true, false>>(x, px, tiles_x, st);
        else rc = last ? start_product<ApplyTask<PAIR, false, true>>(x, px, tiles_x, st) : start_product<ApplyTask<PAIR, false, false>>(x, px, tiles_x, st);
        if (rc) return rc;
    }
    return KT_OK;
}

template <typename T>
int start(StartParams &p, const Plan &plan, bool whole, cudaStream_t st) {
    // a thread takes four pieces at a time; eight CTAs to an SM over all matrices
    const int64_t blocks = (plan.rows * ((plan.cols + 7) / 8) + 1023) / 1024, most = (8 * PRODUCT_SMS + plan.batch - 1) / plan.batch, used = blocks < most ? blocks : most;
    p.sum_blocks = static_cast<int>(used < SUM_BLOCKS ? used : SUM_BLOCKS);
    const dim3 sums(static_cast<unsigned>(p.sum_blocks), static_cast<unsigned>(plan.batch)), grid(static_cast<unsigned>(used), static_cast<unsigned>(plan.batch));
    whole ? k_orth_squares<T, true><<<sums, 256, 0, st>>>(p) : k_orth_squares<T, false><<<sums, 256, 0, st>>>(p);
    KT_CUDA(cudaGetLastError());
    KT_CUDA(launch_behind(whole ? k_orth_start<T, true> : k_orth_start<T, false>, 1, grid, dim3(256), 0, st, p));
    return KT_OK;
}

int check(const char *what, const void *at, const int64_t *stride, int64_t batch, int64_t rows, int64_t cols, int size, bool written) {
    if (at == nullptr) return fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(at) % size) return fail(KT_ERR_ALIGN, "%s is not aligned to its elements", what);
    const int64_t limit = INT64_C(1) << 40;
    if ((rows > 1 && (stride[1] < cols || stride[1] > limit)) || (batch > 1 && (stride[0] < 0 || stride[0] > limit))) return fail(KT_ERR_SHAPE, "%s: strides of %lld and %lld elements", what, (long long)stride[0], (long long)stride[1]);
    if (written && batch > 1) {       // matrices after one another, or rows of all of them in turn
        const int64_t row = rows > 1 ? stride[1] : cols, matrix = (rows - 1) * row + cols;
        if (stride[0] < matrix && !(stride[0] >= cols && row >= (batch - 1) * stride[0] + cols)) return fail(KT_ERR_SHAPE, "%s: matrices of an output overlap (a stride of %lld elements)", what, (long long)stride[0]);
    }
    return KT_OK;
}

constexpr int64_t MAX_SIDE = 1 << 16, MAX_BATCH = 1 << 15;

}  // namespace

int ktd::orth_given_up(unsigned long long *count) {
    KT_CUDA(cudaMemcpyFromSymbol(count, g_waits_given_up, sizeof(*count)));
    return KT_OK;
}

extern "C" {

int64_t kt_orth_workspace(int64_t batch, int64_t rows, int64_t cols) {
    if (batch < 1 || rows < 1 || cols < 1 || batch > MAX_BATCH || rows > MAX_SIDE || cols > MAX_SIDE) return 0;
    return Plan(batch, rows, cols).bytes + 1024;
}

int kt_orth_update(const void *x, const int64_t *x_stride, int dtype, void *out, const int64_t *out_stride, void *workspace, int64_t workspace_bytes, int64_t batch, int64_t rows, int64_t cols,
                   int steps, const float *coefficients, float scale, void *stream) {
    if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_INVALID, "unknown dtype %d", dtype);
    if (batch < 0 || rows < 0 || cols < 0 || batch > MAX_BATCH || rows > MAX_SIDE || cols > MAX_SIDE)
        return fail(KT_ERR_SHAPE, "%lld matrices of %lld x %lld: up to %lld, and %lld to a side, expected", (long long)batch, (long long)rows, (long long)cols, (long long)MAX_BATCH, (long long)MAX_SIDE);
    if (steps < 1 || steps > 64) return fail(KT_ERR_INVALID, "%d steps: 1 to 64 expected", steps);
    if (coefficients == nullptr) return fail(KT_ERR_INVALID, "coefficients is NULL");
    if (!std::isfinite(scale)) return fail(KT_ERR_INVALID, "scale must be finite");
    if (int rc = check_polynomial(steps, coefficients[0], coefficients[1], coefficients[2])) return rc;
    if (batch == 0 || rows == 0 || cols == 0) return KT_OK;
    if (x_stride == nullptr || out_stride == nullptr) return fail(KT_ERR_INVALID, "a stride array is NULL");
    const int size = dtype == KT_F32 ? 4 : 2;
    if (int rc = check("x", x, x_stride, batch, rows, cols, size, false)) return rc;
    if (int rc = check("out", out, out_stride, batch, rows, cols, 2, true)) return rc;
    const Plan plan(batch, rows, cols);
    const int64_t tiles = tiles_of(rows, 128) * tiles_of(cols, 128) * batch;
    if (tiles > INT64_C(1) << 30) return fail(KT_ERR_SHAPE, "batch x rows x cols is too large");
    if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
    if (workspace_bytes < plan.bytes + 1024) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)workspace_bytes, (long long)(plan.bytes + 1024));
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
    char *const ws = reinterpret_cast<char *>(up(reinterpret_cast<intptr_t>(workspace), 1024));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    StartParams p{};
    p.x = x, p.stride[0] = batch > 1 ? x_stride[0] : 0, p.stride[1] = rows > 1 ? x_stride[1] : 0, p.rows = rows, p.cols = cols, p.pitch = plan.pitch_x;
    p.sums = reinterpret_cast<double *>(ws), p.to = reinterpret_cast<__half *>(ws + plan.at_x[0]);
    const int per = 16 / size;
    const bool whole = reinterpret_cast<uintptr_t>(x) % 16 == 0 && p.stride[0] % per == 0 && p.stride[1] % per == 0;
    if (int rc = dtype == KT_F32 ? start<float>(p, plan, whole, st) : start<__nv_bfloat16>(p, plan, whole, st)) return rc;
    // pairs of CTAs where tiles of 256 x 256 give each of them one in the products of symmetric matrices, the smaller ones
    const int64_t symmetric = tiles_of(plan.side, 256);
    const bool pairs = symmetric * (symmetric + 1) / 2 * batch >= PRODUCT_SMS / 2;
    const float a = coefficients[0], b = coefficients[1], c = coefficients[2];
    return pairs ? run<true>(plan, ws, steps, a, b, c, scale, out, out_stride, st) : run<false>(plan, ws, steps, a, b, c, scale, out, out_stride, st);
}

}  // extern "C"
