// kt_orth.cu -- a matrix-shaped update orthogonalised by Newton-Schulz products.  Contract: include/kaitian.h.
//
//   X <- G / |G|_F;  `steps` times  A = X X^T,  X <- (a I + b A + c A^2) X;  out = scale X
// with X^T in place of X where G has more rows than columns, so that A has the shorter side.  The polynomial
// a s + b s^3 + c s^5 takes every singular value s towards one.
//
// Three products a step (kt_product.cuh), in fp16 with fp32 sums: everything that is held between products has a known
// range (singular values of X up to 1.9, of A 3.7, of the factor 7.5 are admitted: kt_orth_update's check of the coefficients; the usual ones
// reach 1.2, 1.5 and a = 3.4), so that fp16's 11 bits can be had where
// bf16, whose range is not needed, has 8: of normal numbers the result is 0.17 to 0.23 % from 64 bits, one in 32 bits rounded to bf16 0.17.
// A rounding of X grows by up to a factor of a a step in the directions that X has little of, so singular values that fall evenly to 10^-3 of
// the largest make it 0.34 to 1.2 %, and few of them beside none more (512 x 512 of rank 64 2.6, of 8 4.3).
// Powers of two keep small entries off fp16's subnormals: X is held times 2^7, A times 2^14, the factor times 2^13 (so that the largest
// admitted A and factor are 60300 and 61440; fp16 ends at 65504).
// A and the factor are symmetric: tiles on and above the diagonal are computed, and written to both sides.
// Every product waits for the one before, so a matrix of few tiles is bound by 15 times what a launch of one takes (256 x 448:
// 79 us, 5 each), and all products in one launch, with a count of arrivals between them, were slower (256 x 384: 110 us where a
// launch to each took 89 then, 74 later: the fences and the count's way through the L2 cost more than a launch).  What fits the shared memory of a CTA or two needs neither
// (below).  4 x 4096 x 2048: some 60 + 41 + 92 us a step, the tensor cores busy
// 76, 55 and 86 % of it (two rounds of 144 tiles on 74 pairs in the first two); power sets the clocks.
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
constexpr int MAX_STEPS = 64;
// Whether the factor's diagonal is kept beyond fp16: where its elements are few, or alike because X is far from square (40 x 5000 with
// and without: 0.17 and 0.31 % off the formula, 30 x 438 0.17 and 0.30; the time of 64 x 640 42 and 36 us).  Elsewhere it changes
// little but for multiples of orthogonal matrices, which are alike too (424 x 424: 0.41 % off).
bool keeps_rest(int64_t side, int64_t length) { return side <= 64 || length >= 8 * side; }
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

// A warp takes 1024 columns of a row, four pieces of eight to a lane; this is the i-th such chunk's row and first column.
struct Chunks {
    uint32_t per_row, all;
    __device__ explicit Chunks(const StartParams &p) : per_row(static_cast<uint32_t>((p.cols + 1023) / 1024)), all(static_cast<uint32_t>(p.rows) * per_row) {}       // 2^22 at most
    __device__ void at(uint32_t i, uint32_t *row, uint32_t *col) const { *row = i / per_row, *col = (i - *row * per_row) * 1024 + threadIdx.x % 32 * 8; }
};

// Sums of squares, 32 at a time in fp32, those in 64 bits.  Where the 32 leave fp32's range, or almost, they are scaled by the power of
// two of the largest before: no element is too large or too small.  (67 MB in 14 us; every element in 64 bits 27.)
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256) k_orth_squares(const StartParams p) {
    __shared__ double of_warp[8];
    let_next_begin();
    const Chunks chunks(p);
    const T *const x = static_cast<const T *>(p.x) + blockIdx.y * p.stride[0];
    double all_of = 0.0;
    for (uint32_t i = blockIdx.x * 8 + threadIdx.x / 32; i < chunks.all; i += gridDim.x * 8) {
        uint32_t row, col;
        chunks.at(i, &row, &col);
        float v[4][8], sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < 4; ++u) read_eight<T, WHOLE>(x + row * p.stride[1], col + u * 256, p.cols, v[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[e % 2] = fmaf(v[u][e], v[u][e], sums[e % 2]);
        const float sum = sums[0] + sums[1];
        if (sum > 0x1p-80f && sum < 0x1p120f) {
            all_of += sum;
            continue;
        }
        float top = 0.0f, scaled = 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[u][e]));
        const uint32_t power = min(__float_as_uint(top) >> 23, 253u);       // an infinity, or a NaN, comes through all the same
        const float by = __uint_as_float((254u - power) << 23);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) scaled = fmaf(v[u][e] * by, v[u][e] * by, scaled);
        all_of += scaled * __longlong_as_double((2 * (static_cast<long long>(power) - 127) + 1023) << 52);
    }
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
    const Chunks chunks(p);
    const uint32_t i = blockIdx.x * 8 + threadIdx.x / 32;
    if (i >= chunks.all) return;
    uint32_t row, col;
    chunks.at(i, &row, &col);
    const T *const x = static_cast<const T *>(p.x) + blockIdx.y * p.stride[0] + row * p.stride[1];
    __half *const to = p.to + (blockIdx.y * p.rows + row) * p.pitch;
    Raw<T, WHOLE> raw[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) raw[u].read(x, col + u * 256, p.cols);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (col + u * 256 >= p.cols) break;
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = narrow ? v[e] * by32 : static_cast<float>(v[e] * by);
        uint4 w;
        w.x = pack_half(v[0], v[1]), w.y = pack_half(v[2], v[3]), w.z = pack_half(v[4], v[5]), w.w = pack_half(v[6], v[7]);
        *reinterpret_cast<uint4 *>(to + col + u * 256) = w;
    }
}

// ------------------------------------------------------------------------------------ products
struct OrthMaps {
    CUtensorMap a, b, out, mirror;
};
enum { GRAM, FACTOR, APPLY, LAST };             // which product

struct OrthParams {
    int rows, cols, side, batch;
    int whole;                                  // both sides of a symmetric result are computed
    int by_copies;                              // the result goes out like the others; else by single elements
    int64_t pitch;                              // of A, in elements
    const __half *gram;
    float *diagonal, *rest;                     // of A; what fp16 leaves of the factor's (rest: NULL where it does not matter); pitch to a matrix
    const __half *x;                            // where rest matters, the X that the factor goes to
    int64_t x_pitch;
    float a, b, c, scale;
    __nv_bfloat16 *out;
    int64_t out_stride[2];
};
__device__ __forceinline__ float2 of_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }       // a pair of fp16

// The factor is computed from the diagonal D of A, kept in fp32, and what is beside it, R, in fp16: A^2 = R^2 + D R + R D + D^2.  The
// diagonal's elements are by far the largest, and alike where X is far from square: their rounding to fp16 would move all singular
// values the same way, and a step takes what is beyond 1.2 four times as far (4 x 465: 0.8 % off the formula, 300 x 3000 0.34; without it
// 0.2).  What is added to the diagonal, in units of the factor:
__device__ __forceinline__ float factor_diagonal(float a, float b, float per_square, float own) { return fmaf(own, fmaf(own, per_square, b * (FACTOR_UNIT / A_UNIT)), a * FACTOR_UNIT); }
// The lane's own of 32 values (a block of 32 rows and columns has its diagonal there).
__device__ __forceinline__ float own_of(const uint32_t (&r)[32]) {
    const int lane = threadIdx.x % 32;
    uint32_t v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = r[i];
#pragma unroll
    for (int n = 16; n; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = lane & n ? v[i + n] : v[i];
    return __uint_as_float(v[0]);
}
__device__ __forceinline__ float beyond_half(float x) { return x - __half2float(__float2half_rn(x)); }
// Eight values at `at` that are the same for a whole warp
struct Eight {
    float4 v[2];
    __device__ explicit Eight(const float *at) { v[0] = reinterpret_cast<const float4 *>(at)[0], v[1] = reinterpret_cast<const float4 *>(at)[1]; }
    __device__ float2 pair(int e) const { return e % 4 == 0 ? make_float2(v[e / 4].x, v[e / 4].y) : make_float2(v[e / 4].z, v[e / 4].w); }
};
// The factor's own diagonal is rounded too, which may count (keeps_rest): what fp16 leaves of it times x is added.
template <typename F>
__device__ __forceinline__ void add_rest(uint32_t (&sums)[32], int at, uint4 x, F rest_of) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float2 f = of_half(w[e / 2]);
        sums[at + e] = __float_as_uint(fmaf(f.x, rest_of(at + e), __uint_as_float(sums[at + e])));
        sums[at + e + 1] = __float_as_uint(fmaf(f.y, rest_of(at + e + 1), __uint_as_float(sums[at + e + 1])));
    }
}

// Three products to a step: A, the factor a I + b A + c A^2 from it, and the next X, factor times X (WIDE) or X times factor.
// A result leaves in boxes of 32 x 32.  The mirrored side of a symmetric one goes through shared memory, where lanes
// are columns: two lanes swap halves, so that each writes two neighbours of one row.  (Two-byte stores straight to memory
// took 27 us to a tile, more than its product.)
template <bool PAIR_, bool WIDE, int KIND>
struct OrthTask {
    using Params = OrthParams;
    using Maps = OrthMaps;
    static constexpr bool PAIR = PAIR_, HALF = true;
    static constexpr int SIDE = PAIR ? 256 : 128, BAND = 8;
    static constexpr bool SYMMETRIC = KIND < APPLY;
    struct Cut {
        int worker, workers, batch, whole, side_tiles, each, tiles_m, tiles_n, steps;
        __device__ Cut(const Params &p, int worker_, int workers_) : worker(worker_), workers(workers_), batch(p.batch), whole(p.whole) {
            side_tiles = (p.side + SIDE - 1) / SIDE;
            tiles_m = (p.rows + SIDE - 1) / SIDE, tiles_n = (p.cols + SIDE - 1) / SIDE;
            each = !SYMMETRIC ? tiles_m * tiles_n : whole ? side_tiles * side_tiles : side_tiles * (side_tiles + 1) / 2;
            steps = ((KIND != GRAM ? p.side : WIDE ? p.cols : p.rows) + K_STEP - 1) / K_STEP;
        }
        __device__ int count() const { return (each * batch - worker + workers - 1) / workers; }
        __device__ Tile tile(int i) const {
            const int at = worker + i * workers, z = at / each;
            int m = 0, n = at - z * each;
            if (!SYMMETRIC) {
                const int band = n / (BAND * tiles_n), left = n - band * BAND * tiles_n, high = min(BAND, tiles_m - band * BAND);
                m = band * BAND + left % high, n = left / high;
            } else if (whole) {
                m = n / side_tiles, n -= m * side_tiles;
            } else {
                for (; n >= side_tiles - m; ++m) n -= side_tiles - m;
                n += m;
            }
            return {m * SIDE, n * SIDE, z, 0, steps, KIND, 0};
        }
    };
    __device__ static bool a_down(const Tile &) { return !WIDE && KIND == GRAM; }
    __device__ static bool b_down(const Tile &) { return WIDE ? !SYMMETRIC : KIND == GRAM; }
    __device__ static const CUtensorMap *map_a(const Maps &maps, const Cut &, const Tile &) { return &maps.a; }
    __device__ static const CUtensorMap *map_b(const Maps &maps, const Cut &, const Tile &) { return &maps.b; }
    __device__ static int rows_a(const Cut &, const Tile &) { return TILE; }
    __device__ static void finish(const Params &p, const Maps &maps, const Cut &, const Tile &t, Part &part) {
        const bool mirrored = SYMMETRIC && !p.whole && t.n != t.m;
        const int rows = SYMMETRIC ? p.side : p.rows, cols = SYMMETRIC ? p.side : p.cols, lane = threadIdx.x % 32;
        if (part.warp_row >= rows) return;
        const float by = KIND == FACTOR ? p.c * (FACTOR_UNIT / A_UNIT / A_UNIT) : KIND == LAST ? p.scale / (FACTOR_UNIT * X_UNIT) : 1.0f / FACTOR_UNIT;
        uint4 g[4] = {};
        // (rows of A are whole vectors, whatever lies past their last element)
        auto of_gram = [&](int c0) {
            if (KIND != FACTOR || part.row >= p.side || c0 >= p.side) return;
            const uint4 *from = reinterpret_cast<const uint4 *>(p.gram + (static_cast<int64_t>(t.z) * p.side + part.row) * p.pitch + c0);
#pragma unroll
            for (int u = 0; u < 4; ++u) g[u] = from[u];
        };
        of_gram(part.col);
        float *const diagonal = p.diagonal + t.z * p.pitch;
        const float per_square = p.c * (FACTOR_UNIT / A_UNIT / A_UNIT), own = KIND == FACTOR && part.row < p.side ? diagonal[part.row] : 0.0f;
        const float per_gram = fmaf(per_square, own, p.b * (FACTOR_UNIT / A_UNIT));
        const bool rest = KIND >= APPLY && p.rest != nullptr && part.row < rows;
        const float rest_of = WIDE && rest ? p.rest[t.z * p.pitch + part.row] : 0.0f;
        over_columns<SIDE / 2>(part, [&](int c0, auto, uint32_t (&r)[32]) {
            if (c0 >= cols) return;
            uint32_t v[16];
            if (rest) {
                const uint4 *const from = reinterpret_cast<const uint4 *>(p.x + (static_cast<int64_t>(t.z) * p.rows + part.row) * p.x_pitch + c0);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint4 x = from[u];
                    add_rest(r, u * 8, x, [&](int e) { return WIDE ? rest_of : p.rest[t.z * p.pitch + c0 + e]; });
                }
            }
#pragma unroll
            for (int e0 = 0; e0 < 32; e0 += 8) {
                const Eight diagonals(KIND == FACTOR ? diagonal + c0 + e0 : diagonal);
#pragma unroll
                for (int e = e0; e < e0 + 8; e += 2) {
                    float2 x = KIND == GRAM ? pair_of(r, e) : mul2(pair_of(r, e), both(by));
                    if constexpr (KIND == FACTOR) {
                        const uint32_t w = e % 8 / 2 == 0 ? g[e / 8].x : e % 8 / 2 == 1 ? g[e / 8].y : e % 8 / 2 == 2 ? g[e / 8].z : g[e / 8].w;
                        x = fma2(of_half(w), fma2(diagonals.pair(e - e0), both(per_square), both(per_gram)), x);
                    }
                    v[e / 2] = KIND == LAST ? pack_bf16(x) : pack_half(x.x, x.y);
                }
            }
            of_gram(c0 + 32);
            if (KIND == LAST && !p.by_copies) {
                if (part.row < rows) {
                    __nv_bfloat16 *const row = p.out + t.z * p.out_stride[0] + part.row * p.out_stride[1] + c0;
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c0 + e < cols) row[e] = __ushort_as_bfloat16(static_cast<unsigned short>(e % 2 ? v[e / 2] >> 16 : v[e / 2] & 0xFFFF));
                }
                return;
            }
            part.store_next();
#pragma unroll
            for (int u = 0; u < 4; ++u)         // rows of 64 bytes, in the 64-byte swizzle
                *reinterpret_cast<uint4 *>(part.store + lane * 64 + ((u ^ (lane / 2 & 3)) << 4)) = make_uint4(v[u * 4], v[u * 4 + 1], v[u * 4 + 2], v[u * 4 + 3]);
            if (SYMMETRIC && c0 == part.warp_row) {       // a block of the diagonal
                const float there = own_of(r), on = KIND == GRAM ? there : fmaf(per_square, there, factor_diagonal(p.a, p.b, per_square, own));
                *reinterpret_cast<__half *>(part.store + lane * 64 + ((lane / 8 ^ (lane / 2 & 3)) << 4) + lane % 8 * 2) = KIND == GRAM ? __half(0.0f) : __float2half_rn(on);
                if (part.row < p.side) {
                    if (KIND == GRAM) diagonal[part.row] = on;
                    else if (p.rest != nullptr) p.rest[t.z * p.pitch + part.row] = beyond_half(on);
                }
            }
            if (mirrored) {
                uint8_t *const mirror = part.store + STORE_BYTES / 2 + (lane & 1) * 64 + (lane & ~1) * 2;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t theirs = __shfl_xor_sync(0xFFFFFFFFu, v[e], 1);
                    *reinterpret_cast<uint32_t *>(mirror + e * 128) = lane & 1 ? (theirs >> 16) | (v[e] & 0xFFFF0000u) : (v[e] & 0xFFFFu) | (theirs << 16);
                }
            }
            part.send(&maps.out, c0, part.warp_row, t.z, false, mirrored ? &maps.mirror : nullptr, STORE_BYTES / 2, part.warp_row, c0);
        });
    }
};

// ------------------------------------------------------------------------------ small matrices
// A matrix whose shorter side fits a tile, and which fits a CTA's shared memory as a whole, goes through all steps in one CTA: X in
// fp16, its shorter side as rows, is an operand as it lies there, along its rows for A and down them for the next X, which takes its
// place two chunks of 64 columns at a time.  Eight warps compute, one thread of the ninth issues the products.  A step of 128 x 640 is
// 6 us: 2.9 of products, 3 of ends between them; reading x, twice, takes 8 us (down the columns of 640 x 128, 25).
// In us, in one CTA and as a launch to a product: 64 x 64 17 and 58, 128 x 128 22 and 67, 128 x 640 50 and 77, 640 x 128 72 and 80, 100 x 333 (by
// elements) 57 and 86, 638 x 126 (so too) 97 and 96, but 117 and 130 with the call; 148 x 128 x 640 52 and 256.  Longer ones do not fit.
constexpr int SMALL_CHUNKS = 10, SMALL_SIDE = TILE, SMALL_LENGTH = SMALL_CHUNKS * 64, SMALL_THREADS = 288, SMALL_READS = 8;
constexpr uint32_t SMALL_A = 0, SMALL_SQUARE = TILE, SMALL_NEXT = 2 * TILE;       // columns of tensor memory: A, A^2, and two places for the next X

struct SmallParams {
    const void *x;
    int64_t x_stride[2], out_stride[2];
    __nv_bfloat16 *out;
    int side, length, steps, whole_out, rest;   // rest: the factor's diagonal beyond fp16 counts
    float a, b, c, scale;
    uint64_t wait_ns;
};
struct SmallSmem {
    alignas(1024) uint8_t x[SMALL_CHUNKS][CHUNK], gram[2][CHUNK], factor[2][CHUNK];
    uint64_t square_full, next_full[2], next_taken[2];
    double sums[8];
    alignas(16) float diagonal[TILE], rest[TILE];       // as in k_product's tasks
    uint32_t tmem;
    Patience waits;
};
// The 16-byte piece `unit` of a row of a chunk, in the 128-byte swizzle.
__device__ __forceinline__ uint4 *piece_of(uint8_t *chunk, int row, int unit) { return reinterpret_cast<uint4 *>(chunk + row * 128 + ((unit ^ (row & 7)) << 4)); }
__device__ __forceinline__ uint32_t *pair_place(uint8_t *chunk, int row, int pair) { return reinterpret_cast<uint32_t *>(piece_of(chunk, row, pair / 4)) + pair % 4; }       // of 32 pairs
__device__ __forceinline__ __half *half_place(uint8_t *chunk, int row, int col) { return reinterpret_cast<__half *>(pair_place(chunk, row, col / 2)) + col % 2; }
__device__ __forceinline__ uint32_t small_word(int n, bool b_down) {
    return (1u << 4) | (b_down ? 1u << 16 : 0u) | (static_cast<uint32_t>(n / 8) << 17) | (static_cast<uint32_t>(TILE / 16) << 24);
}

// The rows of X that a CTA begins with: where they are, how many, how long.
template <typename T>
struct SmallRows {
    const T *x;
    int64_t stride;
    int side, length, chunks;
};
// The i-th eight elements: of memory's rows one after the other, in whole pieces (of 16 bytes, or two such: the length is a multiple of 8);
template <typename T, bool WHOLE, bool WIDE>
struct SmallPiece {
    Raw<T, WHOLE> raw;
    static __device__ int all(const SmallRows<T> &rows) { return rows.side * rows.chunks * 8; }
    static __device__ void place(const SmallRows<T> &rows, int i, int *r, int *unit) { *r = i / (rows.chunks * 8), *unit = i - *r * (rows.chunks * 8); }
    __device__ void read(const SmallRows<T> &rows, int i) {
        int r, unit;
        place(rows, i, &r, &unit);
        const bool there = i < all(rows) && unit * 8 < rows.length;
#pragma unroll
        for (int w = 0; w < static_cast<int>(sizeof(T) / 2); ++w) raw.v[w] = there ? reinterpret_cast<const uint4 *>(rows.x + r * rows.stride + unit * 8)[w] : make_uint4(0, 0, 0, 0);
    }
    __device__ void get(float (&v)[8]) const { raw.get(v); }
    static __device__ void keep(const SmallRows<T> &rows, uint8_t (*to)[CHUNK], int i, const float (&v)[8]) {
        int r, unit;
        place(rows, i, &r, &unit);
        *piece_of(to[unit / 8], r, unit % 8) = make_uint4(pack_half(v[0], v[1]), pack_half(v[2], v[3]), pack_half(v[4], v[5]), pack_half(v[6], v[7]));
    }
};
// by elements, two to a lane of each of four rows;
template <typename T>
struct SmallPiece<T, false, true> {
    T raw[8];
    static __device__ int all(const SmallRows<T> &rows) { return TILE / 4 * rows.chunks * 32; }
    static __device__ void place(const SmallRows<T> &rows, int i, int *r, int *chunk) { *r = i / 32 / rows.chunks * 4, *chunk = i / 32 - *r / 4 * rows.chunks; }
    __device__ void read(const SmallRows<T> &rows, int i) {
        int r, chunk;
        place(rows, i, &r, &chunk);
        const int c = chunk * 64 + i % 32 * 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) raw[e] = i < all(rows) && r + e / 2 < rows.side && c + e % 2 < rows.length ? rows.x[(r + e / 2) * rows.stride + c + e % 2] : static_cast<T>(0.0f);
    }
    __device__ void get(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(raw[e]);
    }
    static __device__ void keep(const SmallRows<T> &rows, uint8_t (*to)[CHUNK], int i, const float (&v)[8]) {
        int r, chunk;
        place(rows, i, &r, &chunk);
#pragma unroll
        for (int e = 0; e < 8; e += 2) *pair_place(to[chunk], r + e / 2, i % 32) = r + e / 2 < rows.side ? pack_half(v[e], v[e + 1]) : 0;
    }
};
// or, where memory's rows are the shorter side (X's columns), in whole pieces again, lanes on one row each after the other,
template <typename T>
struct SmallPiece<T, true, false> {
    Raw<T, true> raw;
    static __device__ int all(const SmallRows<T> &rows) { return rows.side / 8 * rows.chunks * 64; }
    static __device__ void place(const SmallRows<T> &rows, int i, int *r, int *c) { *r = i / (rows.chunks * 64) * 8, *c = i - *r / 8 * (rows.chunks * 64); }
    __device__ void read(const SmallRows<T> &rows, int i) {
        int r, c;
        place(rows, i, &r, &c);
        const bool there = i < all(rows) && c < rows.length;
#pragma unroll
        for (int w = 0; w < static_cast<int>(sizeof(T) / 2); ++w) raw.v[w] = there ? reinterpret_cast<const uint4 *>(rows.x + c * rows.stride + r)[w] : make_uint4(0, 0, 0, 0);
    }
    __device__ void get(float (&v)[8]) const { raw.get(v); }
    static __device__ void keep(const SmallRows<T> &rows, uint8_t (*to)[CHUNK], int i, const float (&v)[8]) {
        int r, c;
        place(rows, i, &r, &c);
#pragma unroll
        for (int e = 0; e < 8; ++e) *half_place(to[c / 64], r + e, c % 64) = __float2half_rn(v[e]);
    }
};
// or by elements of rows (of X, to a multiple of 32) next to each other.
template <typename T>
struct SmallPiece<T, false, false> {
    T raw[8];
    static __device__ int across(const SmallRows<T> &rows) { return (rows.side + 31) & ~31; }
    static __device__ int all(const SmallRows<T> &rows) { return across(rows) * rows.chunks * 8; }
    static __device__ void place(const SmallRows<T> &rows, int i, int *r, int *unit) { *unit = i / across(rows), *r = i - *unit * across(rows); }
    __device__ void read(const SmallRows<T> &rows, int i) {
        int r, unit;
        place(rows, i, &r, &unit);
#pragma unroll
        for (int e = 0; e < 8; ++e) raw[e] = r < rows.side && unit * 8 + e < rows.length ? rows.x[(unit * 8 + e) * rows.stride + r] : static_cast<T>(0.0f);
    }
    __device__ void get(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(raw[e]);
    }
    static __device__ void keep(const SmallRows<T> &rows, uint8_t (*to)[CHUNK], int i, const float (&v)[8]) {
        int r, unit;
        place(rows, i, &r, &unit);
        *piece_of(to[unit / 8], r, unit % 8) = r < rows.side ? make_uint4(pack_half(v[0], v[1]), pack_half(v[2], v[3]), pack_half(v[4], v[5]), pack_half(v[6], v[7])) : make_uint4(0, 0, 0, 0);
    }
};
// Threads next to each other take neighbours in memory: pieces of eight columns of a row, or rows.  A thread's pieces are THREADS
// apart; READS are asked for at once: one after the other they took half of the whole time.
template <typename T, bool WHOLE, bool WIDE, int THREADS, int READS>
__device__ __forceinline__ double small_squares(const SmallRows<T> &rows) {
    double sum = 0.0;
    const int all = SmallPiece<T, WHOLE, WIDE>::all(rows);
    for (int i = threadIdx.x; i < all; i += READS * THREADS) {
        SmallPiece<T, WHOLE, WIDE> piece[READS];
#pragma unroll
        for (int u = 0; u < READS; ++u) piece[u].read(rows, i + u * THREADS);
        float2 adds = both(0.0f);
        float v[8], top = 0.0f;
#pragma unroll
        for (int u = 0; u < READS; ++u) {
            piece[u].get(v);
#pragma unroll
            for (int e = 0; e < 8; e += 2) adds = fma2(make_float2(v[e], v[e + 1]), make_float2(v[e], v[e + 1]), adds);
        }
        const float add = adds.x + adds.y;
        if (add > 0x1p-80f && add < 0x1p120f) {
            sum += add;
            continue;
        }
#pragma unroll
        for (int u = 0; u < READS; ++u) {       // as in k_orth_squares
            piece[u].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
        }
        const uint32_t power = min(__float_as_uint(top) >> 23, 253u);
        const float by = __uint_as_float((254u - power) << 23);
        float scaled = 0.0f;
#pragma unroll
        for (int u = 0; u < READS; ++u) {
            piece[u].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) scaled = fmaf(v[e] * by, v[e] * by, scaled);
        }
        sum += scaled * __longlong_as_double((2 * (static_cast<long long>(power) - 127) + 1023) << 52);
    }
    return sum;
}
// X = G / |G| in fp16, and zeros in rows past the last.
template <typename T, bool WHOLE, bool WIDE, int THREADS, int READS>
__device__ __forceinline__ void small_start(const SmallRows<T> &rows, double sum, uint8_t (*to)[CHUNK]) {
    using Piece = SmallPiece<T, WHOLE, WIDE>;
    const double by = sum == 0.0 ? 0.0 : isfinite(sum) ? X_UNIT / sqrt(sum) : __longlong_as_double(0x7FF8000000000000ll);
    const int power = isfinite(sum) && sum != 0.0 ? ilogb(by) / 2 : 0;       // fp32 need not hold the factor: in two parts it does
    const float by_power = __uint_as_float(static_cast<uint32_t>(power + 127) << 23), by_rest = static_cast<float>(ldexp(by, -power));
    const int all = Piece::all(rows);
    for (int i = threadIdx.x + all; i < TILE * rows.chunks * 8; i += THREADS) *piece_of(to[i / 8 % rows.chunks], i / 8 / rows.chunks, i % 8) = make_uint4(0, 0, 0, 0);
    for (int i = threadIdx.x; i < all; i += READS * THREADS) {
        Piece piece[READS];
#pragma unroll
        for (int u = 0; u < READS; ++u) piece[u].read(rows, i + u * THREADS);
#pragma unroll
        for (int u = 0; u < READS; ++u) {
            if (i + u * THREADS >= all) break;
            float v[8];
            piece[u].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] * by_power * by_rest;       // (by_rest may be NaN)
            Piece::keep(rows, to, i + u * THREADS, v);
        }
    }
}
// 32 values of the factor's row but for the diagonal's: first what A gives, from the row's element of A's diagonal and those of the
// columns, then what R^2 does.  (All at once would be too many registers.)
__device__ __forceinline__ void small_of_gram(const SmallParams &p, uint32_t (&gram)[32], float own, const float *diagonal) {
    const float per_square = p.c * (FACTOR_UNIT / A_UNIT / A_UNIT), per_gram = fmaf(per_square, own, p.b * (FACTOR_UNIT / A_UNIT));
#pragma unroll
    for (int e0 = 0; e0 < 32; e0 += 8) {
        const Eight diagonals(diagonal + e0);
#pragma unroll
        for (int e = e0; e < e0 + 8; e += 2) {
            const float2 f = mul2(pair_of(gram, e), fma2(diagonals.pair(e - e0), both(per_square), both(per_gram)));
            gram[e] = __float_as_uint(f.x), gram[e + 1] = __float_as_uint(f.y);
        }
    }
}
__device__ __forceinline__ void small_factor(const SmallParams &p, const uint32_t (&of_gram)[32], const uint32_t (&square)[32], uint32_t (&v)[16]) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        const float2 f = fma2(pair_of(square, e), both(p.c * (FACTOR_UNIT / A_UNIT / A_UNIT)), pair_of(of_gram, e));
        v[e / 2] = pack_half(f.x, f.y);
    }
}
// The factor's element of the diagonal
__device__ __forceinline__ float small_diagonal(const SmallParams &p, float own, float square) {
    const float per_square = p.c * (FACTOR_UNIT / A_UNIT / A_UNIT);
    return fmaf(per_square, square, factor_diagonal(p.a, p.b, per_square, own));
}
__device__ __forceinline__ void small_half(const uint32_t (&sums)[32], float by, uint32_t (&v)[16]) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        const float2 f = mul2(pair_of(sums, e), both(by));
        v[e / 2] = pack_half(f.x, f.y);
    }
}
// 32 columns of a row as fp16 to half of a chunk
__device__ __forceinline__ void small_keep(uint8_t *chunk, int row, int half, const uint32_t (&v)[16]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) *piece_of(chunk, row, half * 4 + u) = make_uint4(v[u * 4], v[u * 4 + 1], v[u * 4 + 2], v[u * 4 + 3]);
}
// 32 columns of a row of the result: to memory, of a tall matrix (lanes are neighbours) or in whole pieces of 16 bytes, or else to
// half of a chunk, from where small_rows_out takes it.
template <bool WIDE>
__device__ __forceinline__ void small_out(const SmallParams &p, __nv_bfloat16 *out, int side, int row, int c0, const uint32_t (&sums)[32], uint8_t *chunk) {
    const float to_out = p.scale / (FACTOR_UNIT * X_UNIT);
    if (WIDE) {
        uint32_t v[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) v[e / 2] = pack_bf16(mul2(pair_of(sums, e), both(to_out)));
        if (!p.whole_out) {
            small_keep(chunk, row, c0 / 32 % 2, v);
        } else if (row < side && c0 < p.length) {
#pragma unroll
            for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4 *>(out + row * p.out_stride[1] + c0 + u * 8) = make_uint4(v[u * 4], v[u * 4 + 1], v[u * 4 + 2], v[u * 4 + 3]);
        }
    } else if (row < side) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (c0 + e < p.length) out[(c0 + e) * p.out_stride[1] + row] = __float2bfloat16_rn(__uint_as_float(sums[e]) * to_out);
    }
}
__device__ __forceinline__ void small_rows_out(const SmallParams &p, __nv_bfloat16 *out, int side, int chunks, uint8_t (*from)[CHUNK]) {
    for (int i = threadIdx.x; i < side * chunks * 32; i += blockDim.x) {
        const int r = i / 32 / chunks, chunk = i / 32 - r * chunks, c = chunk * 64 + i % 32 * 2;
        const uint32_t v = *pair_place(from[chunk], r, i % 32);
        __nv_bfloat16 *const to = out + r * p.out_stride[1] + c;
        if (c < p.length) to[0] = __ushort_as_bfloat16(static_cast<unsigned short>(v));
        if (c + 1 < p.length) to[1] = __ushort_as_bfloat16(static_cast<unsigned short>(v >> 16));
    }
}
// After a wait that gave up: products in flight get two milliseconds to finish; then the result is NaN.
template <bool WIDE>
__device__ __forceinline__ void small_given_up(const SmallParams &p, __nv_bfloat16 *out, int side) {
    const uint64_t start = now_ns();
    for (int i = 0; i < 100000 && now_ns() - start < 2000000; ++i) __nanosleep(1000);
    for (int i = threadIdx.x; i < side * p.length; i += blockDim.x) {
        const int r = i / p.length, c = i - r * p.length;
        out[WIDE ? r * p.out_stride[1] + c : c * p.out_stride[1] + r] = __ushort_as_bfloat16(0x7FFF);
    }
}

template <typename T, bool WHOLE, bool WIDE>
__global__ void __launch_bounds__(SMALL_THREADS, 1) k_orth_small(const SmallParams p) {
    extern __shared__ uint8_t raw[];
    auto &sm = *reinterpret_cast<SmallSmem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, chunks = (p.length + 63) / 64, k_side = p.side <= 64 ? 64 : 128, blocks = (chunks + 1) / 2;
    const T *const x = static_cast<const T *>(p.x) + blockIdx.x * p.x_stride[0];
    __nv_bfloat16 *const out = p.out + blockIdx.x * p.out_stride[0];
    if (tid == 0) {
        bar_init(&sm.square_full, 1);
        for (int i = 0; i < 2; ++i) bar_init(&sm.next_full[i], 1), bar_init(&sm.next_taken[i], 8);
        sm.waits = {p.wait_ns, 0};
        fence_async_smem();
    }
    if (warp == 8) tmem_alloc(&sm.tmem, 512);
    if (tid < TILE) sm.diagonal[tid] = sm.rest[tid] = 0.0f;
    const SmallRows<T> rows{x, p.x_stride[1], p.side, p.length, chunks};
    double sum = warp < 8 ? small_squares<T, WHOLE, WIDE, 256, SMALL_READS>(rows) : 0.0;
#pragma unroll
    for (int far = 16; far; far /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, far);
    if (warp < 8 && lane == 0) sm.sums[warp] = sum;
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    sum = sm.sums[0];
    for (int w = 1; w < 8; ++w) sum += sm.sums[w];
    if (warp < 8) small_start<T, WHOLE, WIDE, 256, SMALL_READS>(rows, sum, sm.x);
    fence_async_smem();
    __syncthreads();

    const uint32_t tmem = sm.tmem, x_at = smem_addr(sm.x), gram_at = smem_addr(sm.gram), factor_at = smem_addr(sm.factor);
    volatile Patience *const waits = &sm.waits;
    const int group = warp / 4, row = warp % 4 * 32 + lane;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16);
    const bool columns = group * 64 < k_side;              // the group has a part of the square matrices
    uint32_t squares = 0, taken = 0;                       // phases so far: of square_full; blocks of the next X
    bool ok = true;
    auto square = [&](uint32_t to, uint32_t at, int stages) {       // D = M M^T of M along its rows, 64 elements to a stage
        for (int k = 0; k < stages * 4; ++k) {
            const uint64_t off = ((k / 4) * CHUNK + (k % 4) * 32) >> 4, w = operand(OPERAND_ALONG, at) + off;
            mma_smem(tmem + to, w, w, small_word(k_side, false), k > 0);
        }
        mma_commit(&sm.square_full);
    };
    for (int step = 0; step < p.steps; ++step) {
        const bool last = step + 1 == p.steps;
        for (int which = 0; which < 2; ++which) {              // A, then the factor
            if (warp == 8) {
                if (elected()) {
                    tmem_fence_after();
                    if (which == 0) square(SMALL_A, x_at, chunks);
                    else square(SMALL_SQUARE, gram_at, k_side / 64);
                }
                __syncwarp();
            } else {
                ok = ok && bar_wait(&sm.square_full, squares & 1, waits);
                tmem_fence_after();
                if (ok && columns)
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        uint32_t r[32], v[16];
                        const int c0 = group * 64 + half * 32;
                        tmem_load32(lanes + SMALL_A + c0, r);
                        tmem_wait_loads(r);
                        if (which == 0) {
                            small_half(r, 1.0f, v);
                        } else {
                            uint32_t square[32];
                            tmem_load32(lanes + SMALL_SQUARE + c0, square);
                            small_of_gram(p, r, sm.diagonal[row], &sm.diagonal[c0]);
                            tmem_wait_loads(square);
                            small_factor(p, r, square, v);
                        }
                        small_keep(which == 0 ? sm.gram[group] : sm.factor[group], row, half, v);
                    }
                if (ok && columns && group == warp % 4 / 2) {       // the block of the diagonal, read once more: its elements and the rest are too many registers at once
                    const int c = warp % 4 * 32;
                    uint32_t r[32];
                    tmem_load32(lanes + (which == 0 ? SMALL_A : SMALL_SQUARE) + c, r);
                    tmem_wait_loads(r);
                    const float there = own_of(r), own = sm.diagonal[row], on = small_diagonal(p, own, there);
                    *half_place(which == 0 ? sm.gram[group] : sm.factor[group], row, c % 64 + lane) = which == 0 ? __half(0.0f) : __float2half_rn(on);
                    if (which == 0) sm.diagonal[row] = there;
                    else sm.rest[row] = beyond_half(on);
                }
                fence_async_smem();
            }
            ++squares;
            tmem_fence_before();
            __syncthreads();
        }
        if (warp == 8) {
            if (elected()) {
                tmem_fence_after();
                for (int j = 0; j < blocks && ok; ++j) {
                    const uint32_t n = taken + j, at = n & 1;
                    if (!(ok = bar_wait_one(&sm.next_taken[at], (n / 2 + 1) & 1, waits))) break;
                    tmem_fence_after();
                    const int width = min(2, chunks - 2 * j) * 64;
                    for (int k = 0; k < k_side / 16; ++k)
                        mma_smem(tmem + SMALL_NEXT + at * TILE, operand(OPERAND_ALONG, factor_at) + (((k / 4) * CHUNK + (k % 4) * 32) >> 4), operand(OPERAND_DOWN, x_at + 2 * j * CHUNK) + ((k * 2048) >> 4),
                                 small_word(width, true), k > 0);
                    mma_commit(&sm.next_full[at]);
                }
            }
            __syncwarp();
        } else {
            for (int j = 0; j < blocks; ++j) {
                const uint32_t n = taken + j, at = n & 1;
                ok = ok && bar_wait(&sm.next_full[at], n / 2 & 1, waits);
                if (!ok) break;
                tmem_fence_after();
                const int chunk = 2 * j + group;
                uint32_t r[2][32];
                __syncwarp();              // rows past the last have skipped the end of the block before
                if (chunk < chunks) {
                    tmem_load32(lanes + SMALL_NEXT + at * TILE + group * 64, r[0]);
                    tmem_load32(lanes + SMALL_NEXT + at * TILE + group * 64 + 32, r[1]);
                    tmem_wait_loads(r);
                }
                tmem_fence_before();
                bar_arrive_warp(&sm.next_taken[at]);
                if (chunk >= chunks) continue;
                const float rest = sm.rest[row];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int c0 = chunk * 64 + half * 32;
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (p.rest) add_rest(r[half], u * 8, *piece_of(sm.x[chunk], row, half * 4 + u), [&](int) { return rest; });
                    if (!last) {
                        uint32_t v[16];
                        small_half(r[half], 1.0f / FACTOR_UNIT, v);
                        small_keep(sm.x[chunk], row, half, v);
                    } else {
                        small_out<WIDE>(p, out, p.side, row, c0, r[half], sm.x[chunk]);
                    }
                }
            }
            fence_async_smem();
        }
        taken += blocks;
        tmem_fence_before();
        __syncthreads();
    }
    if (WIDE && !p.whole_out) small_rows_out(p, out, p.side, chunks, sm.x);
    if (waits->gave_up) {
        __syncthreads();
        small_given_up<WIDE>(p, out, p.side);
        __syncthreads();
    }
    tmem_fence_after();
    if (warp == 8) tmem_free(tmem, 512);
}

// A matrix whose shorter side fits two tiles goes through all steps in a pair of CTAs, where its length fits.  Each has 128 rows
// of X, an operand of A as they lie there; its rows of A, and then of the factor, take their place (X is read no more by then);
// and, for the next X, of which a CTA's part of the operand is half of the columns, every row of every other chunk of 64 columns.
// The sums of all of the next X stay in tensor memory until the products have ended.  Then they go to the rows, and to the CTA's own
// columns; the copy engine brings the other CTA's (15 bytes a cycle between two CTAs, 3300 cycles) while the next A is multiplied.
// A step of 256 x 384 is 10 us: 4.3 of products, the rest ends of 64 columns of a row to a thread, their way to the copies that the
// tensor cores see (0.4 us each), and arrivals from the other CTA (0.3 to 0.5).  Parts of the rows multiplied as they come are slower
// (by 2 us in all): each has to be made visible by itself.  Reading x, twice, takes 7 us.
// In us, in a pair and as a launch to a product: 129 x 129 55 and 89, 256 x 256 56 and 76, 256 x 384 64 and 80, 384 x 256 69 and 80, 250 x 333
// (by elements) 79 and 97, 74 x 256 x 384 67 and 171, 200 x 192 x 192 152 and 267.  Longer ones do not fit.
constexpr int PAIR_CHUNKS = 6, PAIR_BLOCKS = PAIR_CHUNKS / 2, PAIR_SIDE = 2 * TILE, PAIR_LENGTH = PAIR_CHUNKS * 64, PAIR_WARPS = 16, PAIR_THREADS = PAIR_WARPS * 32;
constexpr uint32_t PAIR_A = 0, PAIR_SQUARE = 256, PAIR_NEXT = 0;        // columns of tensor memory; the next X after both have been read

struct PairSmem {
    alignas(1024) uint8_t rows[PAIR_CHUNKS][CHUNK], cols[PAIR_CHUNKS][CHUNK];       // cols: two, of 256 rows, to each of the CTA's chunks of columns
    uint64_t ready, rows_ready, rows_here;                                      // by warps: those of both CTAs (in the first), and of this one
    uint64_t square_full, next_full[PAIR_BLOCKS], cols_full, cols_late, sent;    // late: of chunks that no row of A takes the place of
    double sums[2 * PAIR_WARPS];
    alignas(16) float diagonal[PAIR_SIDE];                                       // of A, as in k_product's tasks
    uint32_t tmem;
    Patience waits;
};
__device__ __forceinline__ uint32_t pair_word(int n, bool b_down) {
    return (1u << 4) | (b_down ? 1u << 16 : 0u) | (static_cast<uint32_t>(n / 8) << 17) | (static_cast<uint32_t>(PAIR_SIDE / 16) << 24);
}
__device__ __forceinline__ void copy_to_cta(uint32_t to, uint32_t from, uint32_t bytes, uint32_t bar) {         // to a CTA of the pair, counted there
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "r"(from), "r"(bytes), "r"(bar) : "memory");
}
// After a wait for arrivals from both CTAs: what was done there before them is seen here.
__device__ __forceinline__ void seen_of_pair(uint64_t *bar, uint32_t parity) {
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t}" ::"r"(smem_addr(bar)), "r"(parity) : "memory");
}

template <typename T, bool WHOLE, bool WIDE>
__global__ void __launch_bounds__(PAIR_THREADS, 1) k_orth_pair(const SmallParams p) {
    extern __shared__ uint8_t raw[];
    auto &sm = *reinterpret_cast<PairSmem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, chunks = (p.length + 63) / 64, blocks = (chunks + 1) / 2, matrix = blockIdx.x / 2;
    const int rank = static_cast<int>(rank_in_pair()), side = min(p.side - rank * TILE, TILE);       // (its rows)
    const T *const x = static_cast<const T *>(p.x) + matrix * p.x_stride[0] + rank * TILE * (WIDE ? p.x_stride[1] : 1);
    __nv_bfloat16 *const out = p.out + matrix * p.out_stride[0] + rank * TILE * (WIDE ? p.out_stride[1] : 1);
    if (tid == 0) {
        bar_init(&sm.ready, 2 * PAIR_WARPS);
        bar_init(&sm.square_full, 1);
        for (int j = 0; j < PAIR_BLOCKS; ++j) bar_init(&sm.next_full[j], 1);
        bar_init(&sm.rows_ready, 2 * PAIR_WARPS);
        bar_init(&sm.rows_here, PAIR_WARPS);
        bar_init(&sm.cols_full, 1);
        bar_init(&sm.cols_late, 1);
        bar_init(&sm.sent, 2);
        sm.waits = {p.wait_ns, 0};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 0) sums_alloc<true>(&sm.tmem, 512);
    constexpr int READS = WHOLE ? 4 : 2;        // more take too many registers by elements
    const SmallRows<T> rows{x, p.x_stride[1], side, p.length, chunks};
    double sum = small_squares<T, WHOLE, WIDE, PAIR_THREADS, READS>(rows);
#pragma unroll
    for (int far = 16; far; far /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, far);
    cluster_sync();             // the other CTA is there
    if (lane < 2) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(address_in(smem_addr(&sm.sums[rank * PAIR_WARPS + warp]), lane)), "d"(sum) : "memory");
    tmem_fence_before();
    cluster_sync();
    tmem_fence_after();
    sum = sm.sums[lane];
#pragma unroll
    for (int far = 16; far; far /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, far);
    small_start<T, WHOLE, WIDE, PAIR_THREADS, READS>(rows, sum, sm.rows);

    const uint32_t tmem = sm.tmem, rows_at = smem_addr(sm.rows), cols_at = smem_addr(sm.cols);
    volatile Patience *const waits = &sm.waits;
    const int group = warp / 4, row = warp % 4 * 32 + lane, k_side = (p.side + 15) / 16;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16);
    const bool issues = warp == 0 && rank == 0;
    uint32_t squares = 0;                       // phases so far
    bool ok = true, copies = true;              // copies: every one so far has come, so that the barrier may be told of more; the other CTA's then stop as well, for want of these
    auto written = [&](uint64_t *bar, uint64_t *here) {        // the warp's part of an operand
        fence_async_smem();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
            arrive_at(address_in(smem_addr(bar), 0));
            if (here != nullptr) bar_arrive(here);
        }
    };
    // One thread, once the operands are there: products, and an arrival in both CTAs.
    auto may_issue = [&](uint64_t *bar, uint32_t parity) {
        if (!bar_wait_one(bar, parity, waits)) return false;
        seen_of_pair(bar, parity);
        tmem_fence_after();
        return true;
    };
    auto square = [&](uint32_t to, int steps) {       // D = M M^T of M along its rows, `steps` times 16 elements
        for (int k = 0; k < steps; ++k) {
            const uint64_t w = operand(OPERAND_ALONG, rows_at) + (((k / 4) * CHUNK + (k % 4) * 32) >> 4);
            multiply<true>(tmem + to, w, w, pair_word(PAIR_SIDE, false), k > 0);
        }
        multiplied<true>(&sm.square_full);
    };
    __syncthreads();
    for (int c = rank; c < chunks; c += 2)
        for (int i = tid; i < static_cast<int>(CHUNK / 16); i += PAIR_THREADS) reinterpret_cast<uint4 *>(sm.cols[c])[i] = reinterpret_cast<const uint4 *>(sm.rows[c])[i];
    written(&sm.rows_ready, &sm.rows_here);
    for (int step = 0;; ++step) {
        const uint32_t parity = step & 1;
        if (issues) {
            if (elected() && may_issue(&sm.rows_ready, parity)) square(PAIR_A, (p.length + 15) / 16);
            __syncwarp();
        }
        // behind A: the rows to the other CTA's columns
        if (warp == 1) {
            if (lane == 0 && copies) {
                const int mine = (chunks + 1 - rank) / 2;        // of the other CTA's rows
                bar_expect(&sm.cols_full, min(mine, 2) * CHUNK);
                bar_expect(&sm.cols_late, max(mine - 2, 0) * CHUNK);
                copies = bar_wait_one(&sm.rows_here, parity, waits);
                for (int c = rank ^ 1; copies && c < chunks; c += 2)
                    copy_to_cta(address_in(smem_addr(sm.cols[c / 2 * 2 + rank]), rank ^ 1), smem_addr(sm.rows[c]), CHUNK, address_in(smem_addr(c < 4 ? &sm.cols_full : &sm.cols_late), rank ^ 1));
                copies = copies && bar_wait_one(&sm.cols_full, parity, waits);
                if (copies)
                    for (int to = 0; to < 2; ++to) arrive_at(address_in(smem_addr(&sm.sent), to));
            }
            __syncwarp();
        }
        for (int which = 0; which < 2; ++which) {              // A, then the factor
            if (which == 1 && issues) {
                if (elected() && may_issue(&sm.ready, 0)) square(PAIR_SQUARE, k_side);
                __syncwarp();
            }
            ok = ok && bar_wait(&sm.square_full, squares & 1, waits);
            seen_of_pair(&sm.square_full, squares & 1);
            ++squares;
            if (which == 0) {       // rows may be written
                ok = ok && bar_wait(&sm.sent, parity, waits);
                seen_of_pair(&sm.sent, parity);
            }
            __syncwarp();
            tmem_fence_after();
            if (ok)
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    uint32_t r[32], v[16];
                    const int c0 = group * 64 + half * 32;
                    tmem_load32(lanes + PAIR_A + c0, r);
                    tmem_wait_loads(r);
                    if (which == 0) {
                        small_half(r, 1.0f, v);
                    } else {
                        uint32_t square[32];
                        tmem_load32(lanes + PAIR_SQUARE + c0, square);
                        small_of_gram(p, r, sm.diagonal[rank * TILE + row], &sm.diagonal[c0]);
                        tmem_wait_loads(square);
                        small_factor(p, r, square, v);
                    }
                    small_keep(sm.rows[group], row, half, v);
                }
            if (ok && group == rank * 2 + warp % 4 / 2) {           // the block of the diagonal, as in k_orth_small
                const int mine = rank * TILE + row;
                uint32_t r[32];
                tmem_load32(lanes + (which == 0 ? PAIR_A : PAIR_SQUARE) + mine - lane, r);
                tmem_wait_loads(r);
                const float there = own_of(r), on = small_diagonal(p, sm.diagonal[mine], there);
                *half_place(sm.rows[group], row, (mine - lane) % 64 + lane) = which == 0 ? __half(0.0f) : __float2half_rn(on);
                if (which == 0)
                    for (int to = 0; to < 2; ++to) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(address_in(smem_addr(&sm.diagonal[mine]), to)), "f"(there) : "memory");
            }
            if (which == 1 && warp == 1 && lane == 0 && copies) copies = bar_wait_one(&sm.cols_late, parity, waits);
            written(&sm.ready, nullptr);
        }
        if (issues) {
            if (elected() && may_issue(&sm.ready, 1))
                for (int j = 0; j < blocks; ++j) {
                    for (int k = 0; k < k_side; ++k)
                        multiply<true>(tmem + PAIR_NEXT + j * 128, operand(OPERAND_ALONG, rows_at) + (((k / 4) * CHUNK + (k % 4) * 32) >> 4), operand(OPERAND_DOWN, cols_at + j * (2 * CHUNK)) + ((k * 2048) >> 4),
                                       pair_word(128, true), k > 0);
                    multiplied<true>(&sm.next_full[j]);
                }
            __syncwarp();
        }
        // Each group has 32 columns of a block of 128.
        auto block = [&](int j, uint32_t (&r)[32]) {
            ok = ok && bar_wait(&sm.next_full[j], parity, waits);
            __syncwarp();
            if (!ok || j * 4 + group >= 2 * chunks) return false;
            tmem_fence_after();
            tmem_load32(lanes + PAIR_NEXT + j * 128 + group * 32, r);
            tmem_wait_loads(r);
            return true;
        };
        if (step + 1 == p.steps) {
#pragma unroll 1
            for (int j = 0; j < blocks; ++j) {
                uint32_t r[32];
                if (block(j, r)) small_out<WIDE>(p, out, side, row, j * 128 + group * 32, r, sm.cols[2 * j + group / 2]);
            }
            break;
        }
        uint32_t v[PAIR_BLOCKS][16];            // held until the last product has read the factor
#pragma unroll
        for (int j = 0; j < PAIR_BLOCKS; ++j) {
            uint32_t r[32];
            if (j < blocks && block(j, r)) small_half(r, 1.0f / FACTOR_UNIT, v[j]);
        }
#pragma unroll
        for (int j = 0; j < PAIR_BLOCKS; ++j) {
            if (!ok || j * 4 + group >= 2 * chunks) break;
            small_keep(sm.rows[2 * j + group / 2], row, group % 2, v[j]);
            if (group / 2 == rank) small_keep(sm.cols[2 * j + rank], row, group % 2, v[j]);
        }
        written(&sm.rows_ready, &sm.rows_here);
    }
    tmem_fence_before();
    cluster_sync();
    uint32_t gave_up;           // here, or in the other CTA, whose rows are in every product
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(gave_up) : "r"(address_in(smem_addr(&sm.waits.gave_up), rank ^ 1)) : "memory");
    if (WIDE && !p.whole_out) small_rows_out(p, out, side, chunks, sm.cols);       // (a block's columns are free when its products have ended)
    __syncthreads();
    if (gave_up | waits->gave_up) small_given_up<WIDE>(p, out, side);
    __syncwarp();
    cluster_sync();             // the other CTA's reads and products here are done
    tmem_fence_after();
    if (warp == 0) sums_free<true>(tmem, 512);
}

// ---------------------------------------------------------------------------------- host side
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct Plan {
    int64_t batch, rows, cols, side, pitch_x, pitch_a;
    bool wide;
    int64_t at_x[2], at_gram, at_factor, at_diagonal, at_rest, bytes;           // the sums of squares come first
    Plan(int64_t b, int64_t r, int64_t c) : batch(b), rows(r), cols(c), side(r < c ? r : c), pitch_x(up(c, 64)), pitch_a(up(side, 64)), wide(r <= c) {
        int64_t at = up(batch * SUM_BLOCKS * 8, 1024);
        for (int64_t &x : at_x) x = at, at += up(batch * rows * pitch_x * 2, 1024);
        at_gram = at, at += up(batch * side * pitch_a * 2, 1024);
        at_factor = at, at += up(batch * side * pitch_a * 2, 1024);
        at_diagonal = at, at += up(batch * pitch_a * 4, 1024);
        at_rest = at, at += up(batch * pitch_a * 4, 1024);
        bytes = at;
    }
};

// The largest singular value that each step can meet, from one on (|G|_F bounds it), tells whether fp16 holds all
// that is kept between products.
int check_polynomial(int steps, float a, float b, float c) {
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return fail(KT_ERR_INVALID, "the coefficients must be finite");
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

template <bool PAIR, bool WIDE>
int run(const Plan &plan, char *ws, OrthParams p, int steps, cudaStream_t st) {
    constexpr int SIDE = PAIR ? 256 : 128;
    const int64_t matrix_x = plan.rows * plan.pitch_x * 2, matrix_a = plan.side * plan.pitch_a * 2, side_tiles = tiles_of(plan.side, SIDE);
    char *const gram = ws + plan.at_gram, *const factor = ws + plan.at_factor;
    const CUtensorMapDataType half = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    OrthMaps of_gram{}, of_factor{}, apply[2]{};          // apply[i]: from buffer i to the other
    CUtensorMap x[2], square, out;
    for (int i = 0; i < 2; ++i) {
        char *const at = ws + plan.at_x[i];
        if (int rc = describe_operand(&x[i], "the workspace", true, !WIDE, at, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x)) return rc;
        if (int rc = describe_operand(WIDE ? &apply[i].b : &apply[i].a, "the workspace", true, WIDE, at, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x)) return rc;
        if (int rc = describe_matrix(&apply[1 - i].out, "the workspace", half, 2, at, plan.cols, plan.rows, plan.batch, plan.pitch_x * 2, matrix_x, 32, 32)) return rc;
        OrthMaps &m = i == 0 ? of_gram : of_factor;
        char *const result = i == 0 ? gram : factor;
        for (bool mirrored : {false, true})
            if (int rc = describe_matrix(mirrored ? &m.mirror : &m.out, "the workspace", half, 2, result, plan.side, plan.side, plan.batch, plan.pitch_a * 2, matrix_a, 32, 32, !mirrored)) return rc;
        if (int rc = describe_operand(&square, "the workspace", true, false, result, plan.side, plan.side, plan.batch, plan.pitch_a * 2, matrix_a)) return rc;
        if (i == 0) of_factor.a = of_factor.b = square;
        else for (OrthMaps &to : apply) (WIDE ? to.a : to.b) = square;
    }
    // the copy engine takes rows and matrices at multiples of 16 bytes, and writes 16 bytes whole where a row ends inside them
    p.by_copies = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && plan.cols % 8 == 0 && (plan.rows == 1 || p.out_stride[1] % 8 == 0) && (plan.batch == 1 || p.out_stride[0] % 8 == 0);
    if (p.by_copies)
        if (int rc = describe_matrix(&out, "out", CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.out, plan.cols, plan.rows, plan.batch, p.out_stride[1] * 2, p.out_stride[0] * 2, 32, 32)) return rc;
    // Where every tile of the whole square gets a worker of its own, mirroring would only make each take longer.
    p.whole = side_tiles * side_tiles * plan.batch <= PRODUCT_SMS / (PAIR ? 2 : 1);
    const int64_t symmetric = (p.whole ? side_tiles * side_tiles : side_tiles * (side_tiles + 1) / 2) * plan.batch, applied = tiles_of(plan.rows, SIDE) * tiles_of(plan.cols, SIDE) * plan.batch;
    for (int i = 0; i < steps; ++i) {
        of_gram.a = of_gram.b = x[i % 2];
        if (int rc = start_product<OrthTask<PAIR, WIDE, GRAM>>(of_gram, p, symmetric, st)) return rc;
        if (int rc = start_product<OrthTask<PAIR, WIDE, FACTOR>>(of_factor, p, symmetric, st)) return rc;
        OrthMaps m = apply[i % 2];
        p.x = reinterpret_cast<const __half *>(ws + plan.at_x[i % 2]);
        if (i + 1 < steps) {
            if (int rc = start_product<OrthTask<PAIR, WIDE, APPLY>>(m, p, applied, st)) return rc;
        } else {
            if (p.by_copies) m.out = out;
            if (int rc = start_product<OrthTask<PAIR, WIDE, LAST>>(m, p, applied, st)) return rc;
        }
    }
    return KT_OK;
}

template <bool PAIR, typename T, bool WHOLE, bool WIDE>
int start_small(const SmallParams &p, int64_t batch, cudaStream_t st) {
    static std::atomic<uint64_t> raised{0};      // a bit for each device on which the kernel's limit has been raised
    constexpr auto kernel = PAIR ? k_orth_pair<T, WHOLE, WIDE> : k_orth_small<T, WHOLE, WIDE>;
    constexpr size_t bytes = (PAIR ? sizeof(PairSmem) : sizeof(SmallSmem)) + 1024;
    static_assert(bytes <= 227 * 1024, "the matrix and its squares have to fit");
    int dev = 0;
    KT_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
        KT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
        raised.fetch_or(bit, std::memory_order_relaxed);
    }
    if constexpr (PAIR) {
        KT_CUDA(launch_joint(kernel, 2, dim3(static_cast<unsigned>(2 * batch)), dim3(PAIR_THREADS), bytes, st, p));
    } else {
        kernel<<<static_cast<unsigned>(batch), SMALL_THREADS, bytes, st>>>(p);
        KT_CUDA(cudaGetLastError());
    }
    return KT_OK;
}
template <bool PAIR, typename T>
int start_small(const SmallParams &p, int64_t batch, bool whole, bool wide, cudaStream_t st) {
    if (!wide) return whole ? start_small<PAIR, T, true, false>(p, batch, st) : start_small<PAIR, T, false, false>(p, batch, st);
    return whole ? start_small<PAIR, T, true, true>(p, batch, st) : start_small<PAIR, T, false, true>(p, batch, st);
}

template <typename T>
int start(StartParams &p, const Plan &plan, bool whole, cudaStream_t st) {
    const int64_t blocks = (plan.rows * ((plan.cols + 1023) / 1024) + 7) / 8;       // eight warps' chunks
    p.sum_blocks = static_cast<int>(blocks < SUM_BLOCKS ? blocks : SUM_BLOCKS);
    const dim3 sums(static_cast<unsigned>(p.sum_blocks), static_cast<unsigned>(plan.batch)), grid(static_cast<unsigned>(blocks), static_cast<unsigned>(plan.batch));
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
    if (steps < 1 || steps > MAX_STEPS) return fail(KT_ERR_INVALID, "%d steps: 1 to %d expected", steps, MAX_STEPS);
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
    const int64_t length = plan.wide ? cols : rows;
    const bool small = plan.side <= SMALL_SIDE && length <= SMALL_LENGTH, pair = plan.side <= PAIR_SIDE && length <= PAIR_LENGTH;
    if (small || pair) {
        SmallParams m{};
        m.x = x, m.out = static_cast<__nv_bfloat16 *>(out), m.side = static_cast<int>(plan.side), m.length = static_cast<int>(length), m.steps = steps;
        m.x_stride[0] = p.stride[0], m.x_stride[1] = p.stride[1], m.out_stride[0] = batch > 1 ? out_stride[0] : 0, m.out_stride[1] = rows > 1 ? out_stride[1] : 0;
        m.whole_out = reinterpret_cast<uintptr_t>(out) % 16 == 0 && m.out_stride[0] % 8 == 0 && m.out_stride[1] % 8 == 0 && length % 32 == 0;
        m.rest = keeps_rest(plan.side, length);
        m.a = coefficients[0], m.b = coefficients[1], m.c = coefficients[2], m.scale = scale, m.wait_ns = wait_limit_ns();
        const bool pieces = whole && cols % 8 == 0;
        if (small) return dtype == KT_F32 ? start_small<false, float>(m, batch, pieces, plan.wide, st) : start_small<false, __nv_bfloat16>(m, batch, pieces, plan.wide, st);
        return dtype == KT_F32 ? start_small<true, float>(m, batch, pieces, plan.wide, st) : start_small<true, __nv_bfloat16>(m, batch, pieces, plan.wide, st);
    }
    if (int rc = dtype == KT_F32 ? start<float>(p, plan, whole, st) : start<__nv_bfloat16>(p, plan, whole, st)) return rc;
    // Pairs of CTAs where there are tiles of 256 x 256 for two thirds of them in the products of symmetric matrices, the smaller ones.
    // In us, one CTA to a tile and pairs: 2048 x 2048 (36 tiles) 243 and 266, 4 x 1024 x 1024 (40) 171 and 196, 16 x 512 x 512 (48)
    // 163 and 159, 20 x 512 x 512 (60) 181 and 185, 12 x 768 x 768 (72) 218 and 215.  Where a side ends early in a tile of 256, which the rule does
    // not look at, pairs lose: 15 x 1000 x 300 (45) 201 and 249.
    const int64_t symmetric = tiles_of(plan.side, 256);
    const bool pairs = symmetric * (symmetric + 1) / 2 * batch >= 45;
    OrthParams q{};
    q.rows = static_cast<int>(rows), q.cols = static_cast<int>(cols), q.side = static_cast<int>(plan.side), q.batch = static_cast<int>(batch);
    q.pitch = plan.pitch_a, q.gram = reinterpret_cast<const __half *>(ws + plan.at_gram), q.x_pitch = plan.pitch_x;
    q.diagonal = reinterpret_cast<float *>(ws + plan.at_diagonal), q.rest = keeps_rest(plan.side, length) ? reinterpret_cast<float *>(ws + plan.at_rest) : nullptr;
    q.a = coefficients[0], q.b = coefficients[1], q.c = coefficients[2], q.scale = scale;
    q.out = static_cast<__nv_bfloat16 *>(out), q.out_stride[0] = out_stride[0], q.out_stride[1] = out_stride[1];
    if (plan.wide) return pairs ? run<true, true>(plan, ws, q, steps, st) : run<false, true>(plan, ws, q, steps, st);
    return pairs ? run<true, false>(plan, ws, q, steps, st) : run<false, false>(plan, ws, q, steps, st);
}

}  // extern "C"
