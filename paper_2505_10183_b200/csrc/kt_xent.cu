// kt_xent.cu -- softmax cross entropy of hidden rows against the weights of a vocabulary, with its gradient, without
// keeping the logits.  Contracts: include/kaitian.h.
//
// With logits l_iv = scale h_i . w_v and lse_i = log sum_v exp(l_iv):
//   forward    loss_i = lse_i - l_{i, t_i}
//   backward   P_iv = scale ((g_i + z_i) exp(l_iv - lse_i) - g_i [v = t_i])  for dloss g and dlse z,
//              dh = P W,  dW = P^T h
// Three kinds of products (kt_product.cuh):
//   loss   a tile of logits becomes a maximum, a sum of exponentials and perhaps the target's logit of each row
//   grad   the logits are formed again, and leave the chip as P in bf16, a piece of the vocabulary at a time (the second
//          products of the tensor cores take 16-bit operands; bf16 because P spans the range of probabilities)
//   dh, dW from the piece.  dW of the piece's rows is whole; dh is summed over the pieces in fp32.
// Rows that do not count are left out before the products: the rows that do are numbered in order, and where any are
// missing their hidden rows are copied next to each other, so what the others hold is never multiplied.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>

#include <atomic>
#include <cmath>

#include "kt_internal.h"
#include "kt_pairs.cuh"
#include "kt_product.cuh"

using namespace ktd;

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int64_t MAX_ROWS = 1 << 20, MAX_VOCAB = 1 << 24, MAX_DIM = 1 << 16;

// What a counted row brings to the products, in the order in which they are numbered.
struct Row {
    int target;                                 // PAST_VOCAB where it is none of the vocabulary's
    float lse2;                                 // in units of log 2
    float both, only;                           // scale (g + z), scale g
};
constexpr int PAST_VOCAB = 0x7FFFFFFF;

__device__ __forceinline__ int round_to(int x, int m) { return (x + m - 1) / m * m; }

// ------------------------------------------------------------------------------ rows that count
struct RowsParams {
    const int64_t *targets;
    const __nv_bfloat16 *hidden;
    int64_t hidden_stride;
    __nv_bfloat16 *packed;                      // counted rows of hidden, where some do not count
    int *count, *index;                         // index[i]: the row that is the i-th to count
    Row *rows;
    const float *dloss, *dlse, *lse;            // backward
    float *loss_out, *lse_out;                  // forward
    __nv_bfloat16 *dhidden;
    int64_t dhidden_stride;
    int n, dim, vocab, each;                    // each: rows to a CTA
    float scale;
};

__device__ __forceinline__ int block_sum(int x, int *shared) {
    x = __reduce_add_sync(0xFFFFFFFFu, x);
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += shared[w];
    return sum;
}

// Every CTA goes over all targets to find out where its own rows begin: a few microseconds for 64 thousand of them
// from the L2, and no CTA waits for another.
__global__ void __launch_bounds__(256) k_xent_rows(const RowsParams p) {
    __shared__ int sums[8], place[256];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    let_next_begin();
    const int begin = min(p.n, static_cast<int>(blockIdx.x) * p.each), end = min(p.n, begin + p.each);
    int before = 0, all = 0;
    for (int i = tid; i < p.n; i += 256) {
        const int counts = p.targets[i] >= 0;
        all += counts;
        if (i < begin) before += counts;
    }
    all = block_sum(all, sums);
    before = block_sum(before, sums);
    const bool copy = all < p.n;
    const int pieces = p.dim / 8;
    if (blockIdx.x == 0) {
        if (tid == 0) *p.count = all;
        if (copy)       // a stage of the reduction over rows may read past the last: zeros there
            for (int i = all * pieces + tid; i < round_to(all, K_STEP) * pieces; i += 256) reinterpret_cast<uint4 *>(p.packed)[i] = make_uint4(0, 0, 0, 0);
    }
    for (int base = begin; base < end; base += 256) {
        const int i = base + tid;
        const int64_t target = i < end ? p.targets[i] : -1;
        const bool counts = target >= 0;
        const unsigned mask = __ballot_sync(0xFFFFFFFFu, counts);
        __syncthreads();
        if (lane == 0) sums[warp] = __popc(mask);
        __syncthreads();
        int at = before + __popc(mask & ((1u << lane) - 1));
        for (int w = 0; w < 8; ++w) {
            if (w < warp) at += sums[w];
            before += sums[w];
        }
        place[tid] = counts ? at : -1;
        if (counts) {
            const bool known = target < p.vocab;
            Row row{known ? static_cast<int>(target) : PAST_VOCAB, 0.0f, 0.0f, 0.0f};
            if (p.lse != nullptr) {
                const float g = known ? p.dloss[i] : __int_as_float(0x7FFFFFFF), z = p.dlse != nullptr ? p.dlse[i] : 0.0f;
                row.lse2 = p.lse[i] * LOG2E, row.both = (g + z) * p.scale, row.only = g * p.scale;
            }
            p.rows[at] = row, p.index[at] = i;
        } else if (i < end && p.loss_out != nullptr) {
            p.loss_out[i] = 0.0f, p.lse_out[i] = 0.0f;
        }
        if (!copy) continue;
        __syncthreads();
        for (int r = warp; r < min(256, end - base); r += 8) {
            const int to = place[r];
            if (to >= 0) {
                const uint4 *from = reinterpret_cast<const uint4 *>(p.hidden + (base + r) * p.hidden_stride);
                uint4 *const row = reinterpret_cast<uint4 *>(p.packed + static_cast<int64_t>(to) * p.dim);
                for (int c = lane; c < pieces; c += 32) row[c] = from[c];
            } else if (p.dhidden != nullptr) {
                uint4 *const row = reinterpret_cast<uint4 *>(p.dhidden + (base + r) * p.dhidden_stride);
                for (int c = lane; c < pieces; c += 32) row[c] = make_uint4(0, 0, 0, 0);
            }
        }
    }
}

// ------------------------------------------------------------------------------------ products
// The order of tiles: bands of up to `band` tiles of rows, in a band column after column, so that the tiles
// in work at one time share rows and columns that the L2 holds.
__device__ __forceinline__ void in_bands(int i, int tiles_m, int tiles_n, int band, int *m, int *n) {
    band = min(band, tiles_m);
    const int per_band = band * tiles_n, b = i / per_band, in = i - b * per_band, high = min(band, tiles_m - b * band);
    *n = in / high;
    *m = b * band + in - *n * high;
}

struct LogitsParams {
    const int *count;
    const Row *rows;
    float2 *parts;                              // [tiles of columns][n]: maximum (units of log 2) and sum
    float *at_target;                           // the target's logit (units of log 2)
    int n, vocab, steps, from, past, band;      // columns from ... past of the vocabulary
    float scale_log2;
};

template <bool PAIR_>
struct LogitsTask {
    using Params = LogitsParams;
    static constexpr bool PAIR = PAIR_, A_DOWN = false, B_DOWN = false, HALF = false;
    static constexpr int SIDE = PAIR ? 256 : 128;
    __device__ static int tiles_m(const Params &p) { return (*p.count + SIDE - 1) / SIDE; }
    __device__ static int tiles(const Params &p) { return tiles_m(p) * ((p.past - p.from + SIDE - 1) / SIDE); }
    __device__ static bool second_a(const Params &p) { return *p.count < p.n; }
    __device__ static bool second_b(const Params &) { return false; }
    __device__ static Tile tile(const Params &p, int i) {
        int m, n;
        in_bands(i, tiles_m(p), (p.past - p.from + SIDE - 1) / SIDE, p.band, &m, &n);
        return {m * SIDE, p.from + n * SIDE, 0, 0, p.steps, 0};
    }
};

template <bool PAIR_>
struct LossTask : LogitsTask<PAIR_> {
    using Base = LogitsTask<PAIR_>;
    __device__ static void finish(const LogitsParams &p, const ProductMaps &, const Tile &t, const Part &part) {
        const bool counts = part.row < *p.count;
        const int target = counts ? p.rows[part.row].target : -1;
        float top = -INFINITY, sum = 0.0f;
        over_columns<Base::SIDE>(part, [&](int c, uint32_t (&r)[32]) {
            const int v0 = t.n + c;
            if (v0 >= p.vocab) return;
            if (v0 + 32 > p.vocab)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (v0 + e >= p.vocab) r[e] = __float_as_uint(-INFINITY);
            float high[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) high[e] = __uint_as_float(r[e]);
#pragma unroll
            for (int e = 4; e < 32; ++e) high[e % 4] = fmaxf(high[e % 4], __uint_as_float(r[e]));
            const float m = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3])) * p.scale_log2;
            if (m > top) sum *= exp2_fast(top - m), top = m;
            const float shift = top == -INFINITY ? 0.0f : -top;
            float2 add[2] = {both(0.0f), both(0.0f)};
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 x = fma2(pair_of(r, e), both(p.scale_log2), both(shift));
                add[e / 2 % 2] = add2(add[e / 2 % 2], make_float2(exp2_fast(x.x), exp2_fast(x.y)));
            }
            add[0] = add2(add[0], add[1]);
            sum += add[0].x + add[0].y;
            const int d = target - v0;
            if (static_cast<unsigned>(d) < 32u) {
                float x = 0.0f;
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e == d) x = __uint_as_float(r[e]);
                p.at_target[part.row] = x * p.scale_log2;
            }
        });
        if (counts) p.parts[static_cast<int64_t>(t.n / Base::SIDE) * p.n + part.row] = make_float2(top, sum);
    }
};

// 64 columns of a row, as 16-bit values, through the store to a matrix.
template <typename F>
__device__ __forceinline__ void pack_row(const Part &part, int c, F value) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint4 v;
        v.x = pack_bf16(value(u * 8), value(u * 8 + 1)), v.y = pack_bf16(value(u * 8 + 2), value(u * 8 + 3));
        v.z = pack_bf16(value(u * 8 + 4), value(u * 8 + 5)), v.w = pack_bf16(value(u * 8 + 6), value(u * 8 + 7));
        *part.piece((c % 64) / 8 + u) = v;
    }
}

template <bool PAIR_>
struct GradTask : LogitsTask<PAIR_> {
    using Base = LogitsTask<PAIR_>;
    __device__ static void finish(const LogitsParams &p, const ProductMaps &maps, const Tile &t, const Part &part) {
        const int count = *p.count;
        if (part.warp_row >= round_to(count, TILE)) return;
        const bool counts = part.row < count;
        const Row row = counts ? p.rows[part.row] : Row{-1, 0.0f, 0.0f, 0.0f};
        over_columns<Base::SIDE>(part, [&](int c, uint32_t (&r)[32]) {
            const int v0 = t.n + c;
            if (v0 - c % 64 >= p.past) return;
            if (c % 64 == 0) part.store_free();
            const int d = row.target - v0, left = p.past - v0;
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 y = fma2(pair_of(r, e), both(p.scale_log2), both(-row.lse2));
                const float2 g = mul2(make_float2(exp2_fast(y.x), exp2_fast(y.y)), both(row.both));
                x[e] = g.x, x[e + 1] = g.y;
            }
            if (static_cast<unsigned>(d) < 32u)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e == d) x[e] -= row.only;
            if (!counts || left < 32)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (!counts || e >= left) x[e] = 0.0f;
            pack_row(part, c, [&](int e) { return x[e]; });
            if (c % 64 == 32) part.send(&maps.out, v0 - 32 - p.from, part.warp_row, 0);
        });
    }
};

// dW of a piece: [columns of the piece] x [dim], reduced over the counted rows.
struct WeightParams {
    const int *count;
    int n, tiles_m, tiles_n, band, vocab, dim, from;
};
template <bool PAIR_>
struct WeightTask {
    using Params = WeightParams;
    static constexpr bool PAIR = PAIR_, A_DOWN = true, B_DOWN = true, HALF = false;
    static constexpr int SIDE = PAIR ? 256 : 128;
    __device__ static int tiles(const Params &p) { return p.tiles_m * p.tiles_n; }
    __device__ static bool second_a(const Params &) { return false; }
    __device__ static bool second_b(const Params &p) { return *p.count < p.n; }
    __device__ static Tile tile(const Params &p, int i) {
        int m, n;
        in_bands(i, p.tiles_m, p.tiles_n, p.band, &m, &n);
        return {m * SIDE, n * SIDE, 0, 0, (*p.count + K_STEP - 1) / K_STEP, 0};
    }
    __device__ static void finish(const Params &p, const ProductMaps &maps, const Tile &t, const Part &part) {
        if (p.from + part.warp_row >= p.vocab) return;
        over_columns<SIDE>(part, [&](int c, uint32_t (&r)[32]) {
            if (t.n + c - c % 64 >= p.dim) return;
            if (c % 64 == 0) part.store_free();
            pack_row(part, c, [&](int e) { return __uint_as_float(r[e]); });
            if (c % 64 == 32) part.send(&maps.out, t.n + c - 32, p.from + part.warp_row, 0);
        });
    }
};

// dh of a piece, reduced over a share of its columns: added to, or the first of, the share's own sums; or (to != NULL)
// all there is, to the rows themselves.  (The description of W begins with the piece's first row.)
struct HiddenParams {
    const int *count, *index;
    __nv_bfloat16 *to;
    int64_t to_stride;
    int tiles_n, band, dim, shares, steps, add;       // steps of the piece
};
template <bool PAIR_>
struct HiddenTask {
    using Params = HiddenParams;
    static constexpr bool PAIR = PAIR_, A_DOWN = false, B_DOWN = true, HALF = false;
    static constexpr int SIDE = PAIR ? 256 : 128;
    __device__ static int tiles_m(const Params &p) { return (*p.count + SIDE - 1) / SIDE; }
    __device__ static int tiles(const Params &p) { return tiles_m(p) * p.tiles_n * p.shares; }
    __device__ static bool second_a(const Params &) { return false; }
    __device__ static bool second_b(const Params &) { return false; }
    __device__ static Tile tile(const Params &p, int i) {
        int m, n;
        const int share = i % p.shares, begin = static_cast<int>(static_cast<int64_t>(p.steps) * share / p.shares), end = static_cast<int>(static_cast<int64_t>(p.steps) * (share + 1) / p.shares);
        in_bands(i / p.shares, tiles_m(p), p.tiles_n, p.band, &m, &n);
        return {m * SIDE, n * SIDE, 0, begin * K_STEP, end - begin, share};
    }
    __device__ static void finish(const Params &p, const ProductMaps &maps, const Tile &t, const Part &part) {
        const int count = *p.count;
        if (part.warp_row >= count) return;
        __nv_bfloat16 *const row = p.to != nullptr && part.row < count ? p.to + p.index[part.row] * p.to_stride : nullptr;
        over_columns<SIDE>(part, [&](int c, uint32_t (&r)[32]) {
            const int c0 = t.n + c;
            if (c0 >= p.dim) return;
            if (p.to != nullptr) {
                if (row != nullptr)
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (c0 + e < p.dim) {
                            uint4 v;
                            v.x = pack_bf16(pair_of(r, e)), v.y = pack_bf16(pair_of(r, e + 2)), v.z = pack_bf16(pair_of(r, e + 4)), v.w = pack_bf16(pair_of(r, e + 6));
                            *reinterpret_cast<uint4 *>(row + c0 + e) = v;
                        }
                return;
            }
            part.store_free();
#pragma unroll
            for (int u = 0; u < 8; ++u) *part.piece(u) = make_uint4(r[u * 4], r[u * 4 + 1], r[u * 4 + 2], r[u * 4 + 3]);
            part.send(&maps.out, c0, part.warp_row, t.share, p.add != 0);
        });
    }
};

// ------------------------------------------------------------------------------------- ends
// The parts of a row joined; 8 rows to a CTA, 32 threads to a row.
__global__ void __launch_bounds__(256) k_xent_join(const int *count, const int *index, const Row *rows, const float2 *parts, const float *at_target, int n, int tiles, float *loss, float *lse) {
    __shared__ float2 of_warp[8][8];
    let_next_begin();
    after_previous();
    const int tid = threadIdx.x, r = tid % 8, row = blockIdx.x * 8 + r;
    const bool counts = row < *count;
    float top = -INFINITY, sum = 0.0f;
    auto join = [&](float2 x) {
        const float high = fmaxf(top, x.x), zero = high == -INFINITY ? 0.0f : high;
        sum = sum * exp2f(top - zero) + x.y * exp2f(x.x - zero);
        top = high;
    };
    if (counts)
#pragma unroll 4
        for (int i = tid / 8; i < tiles; i += 32) join(parts[static_cast<int64_t>(i) * n + row]);
#pragma unroll
    for (int far = 8; far < 32; far *= 2) join(make_float2(__shfl_xor_sync(0xFFFFFFFFu, top, far), __shfl_xor_sync(0xFFFFFFFFu, sum, far)));
    if (tid % 32 < 8) of_warp[tid / 32][r] = make_float2(top, sum);
    __syncthreads();
    if (tid >= 8 || !counts) return;
    top = -INFINITY, sum = 0.0f;
    for (int w = 0; w < 8; ++w) join(of_warp[w][r]);
    const float high = log2f(sum);
    const int i = index[row];
    lse[i] = (top + high) * LN2;
    // the maximum and the target's logit first: they are close where the loss is small
    loss[i] = rows[row].target == PAST_VOCAB ? __int_as_float(0x7FFFFFFF) : ((top - at_target[row]) + high) * LN2;
}

// The shares of dh added up, in order.
__global__ void __launch_bounds__(256) k_xent_dhidden(const int *count, const int *index, const float *sums, int shares, int64_t share, int dim, __nv_bfloat16 *to, int64_t stride) {
    let_next_begin();
    after_previous();
    const int pieces = dim / 8, all = *count;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < static_cast<int64_t>(all) * pieces; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int row = static_cast<int>(i / pieces), c = static_cast<int>(i - static_cast<int64_t>(row) * pieces) * 8;
        const float *from = sums + static_cast<int64_t>(row) * dim + c;
        float4 a = *reinterpret_cast<const float4 *>(from), b = *reinterpret_cast<const float4 *>(from + 4);
        for (int s = 1; s < shares; ++s) {
            const float4 c0 = *reinterpret_cast<const float4 *>(from + s * share), c1 = *reinterpret_cast<const float4 *>(from + s * share + 4);
            a.x += c0.x, a.y += c0.y, a.z += c0.z, a.w += c0.w, b.x += c1.x, b.y += c1.y, b.z += c1.z, b.w += c1.w;
        }
        uint4 v;
        v.x = pack_bf16(a.x, a.y), v.y = pack_bf16(a.z, a.w), v.z = pack_bf16(b.x, b.y), v.w = pack_bf16(b.z, b.w);
        *reinterpret_cast<uint4 *>(to + index[row] * stride + c) = v;
    }
}

// ---------------------------------------------------------------------------------- host side
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
int64_t tiles_of(int64_t x, int side) { return (x + side - 1) / side; }

// Whether a product of m x n results is worked on by pairs of CTAs: where tiles of 256 x 256 give every pair
// at least one.
bool by_pairs(int64_t m, int64_t n) { return tiles_of(m, 256) * tiles_of(n, 256) >= PRODUCT_SMS / 2; }

constexpr int64_t PIECE_BYTES = INT64_C(512) << 20;        // of P, at most

// Where everything lies in the workspace, and how the work is cut: from the sizes alone.
struct Plan {
    int64_t n, dim, vocab;
    bool backward;
    int64_t piece, pieces, shares;              // columns of the vocabulary to a piece; shares of dh's reduction
    bool pairs_logits, pairs_hidden, pairs_weight;
    int64_t at_index, at_rows, at_packed, at_parts, at_target, at_p, at_sums, bytes;
    Plan(int64_t rows, int64_t dims, int64_t words, bool back) : n(rows), dim(dims), vocab(words), backward(back) {
        int64_t at = 0;
        auto take = [&](int64_t size) {
            const int64_t here = at;
            at += up(size, 1024);
            return here;
        };
        take(4);                                // the number of rows that count
        at_index = take(4 * n), at_rows = take(static_cast<int64_t>(sizeof(Row)) * n);
        at_packed = take(2 * up(n, K_STEP) * dim);
        const int64_t room = PIECE_BYTES / (2 * up(n, TILE)) / 256 * 256, most = room < 256 ? 256 : room;
        pieces = backward ? tiles_of(vocab, static_cast<int>(most)) : 1;
        piece = backward ? up((vocab + pieces - 1) / pieces, 256) : vocab;
        pieces = (vocab + piece - 1) / piece;
        pairs_logits = by_pairs(n, piece), pairs_hidden = by_pairs(n, dim), pairs_weight = by_pairs(piece, dim);
        // dh: few tiles share the reduction over the vocabulary among several CTAs, at least 16 stages to each
        const int side = pairs_hidden ? 256 : 128;
        const int64_t tiles = tiles_of(n, side) * tiles_of(dim, side), places = PRODUCT_SMS / (pairs_hidden ? 2 : 1), steps = (piece + K_STEP - 1) / K_STEP;
        shares = places / tiles;
        if (shares > steps / 16) shares = steps / 16;
        if (shares < 1) shares = 1;
        at_parts = take(backward ? 0 : 8 * n * tiles_of(vocab, pairs_logits ? 256 : 128)), at_target = take(backward ? 0 : 4 * n);
        at_p = take(backward ? 2 * up(n, TILE) * piece : 0);
        at_sums = take(backward && (pieces > 1 || shares > 1) ? 4 * shares * n * dim : 0);
        bytes = at;
    }
};

int check_matrix(const char *what, const void *at, int64_t stride, int64_t rows, int64_t dim) {
    if (at == nullptr) return fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(at) % 16) return fail(KT_ERR_ALIGN, "%s is not 16-byte aligned", what);
    if (rows <= 1) return KT_OK;
    if (stride % 8) return fail(KT_ERR_ALIGN, "%s: the stride of its rows must be a multiple of 8 elements", what);
    if (stride < dim || stride >= INT64_C(1) << 38) return fail(KT_ERR_SHAPE, "%s: rows of %lld elements cannot be %lld apart", what, (long long)dim, (long long)stride);
    return KT_OK;
}
int check_vector(const char *what, const void *at, size_t size, bool optional = false) {
    if (at == nullptr) return optional ? KT_OK : fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(at) % size) return fail(KT_ERR_ALIGN, "%s is not aligned to its elements", what);
    return KT_OK;
}
int check_common(int64_t rows, int64_t dim, int64_t vocab, int dtype, float scale) {
    if (dtype != KT_BF16) return fail(KT_ERR_INVALID, "the loss takes KT_BF16 rows and weights");
    if (rows < 0 || rows > MAX_ROWS) return fail(KT_ERR_SHAPE, "%lld rows: 0 to %lld expected", (long long)rows, (long long)MAX_ROWS);
    if (dim < 8 || dim % 8 || dim > MAX_DIM) return fail(KT_ERR_SHAPE, "dim %lld: a multiple of 8 up to %lld expected", (long long)dim, (long long)MAX_DIM);
    if (vocab < 1 || vocab > MAX_VOCAB) return fail(KT_ERR_SHAPE, "a vocabulary of %lld: 1 to %lld expected", (long long)vocab, (long long)MAX_VOCAB);
    if (!(scale >= 1.0f / (1 << 20)) || !(scale <= 1 << 20)) return fail(KT_ERR_INVALID, "scale must be from 2^-20 to 2^20");
    return KT_OK;
}
int check_workspace(const void *workspace, int64_t bytes, int64_t need) {
    if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
    if (bytes < need) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)bytes, (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
    return KT_OK;
}

int start_rows(RowsParams &q, const Plan &plan, char *ws, cudaStream_t st) {
    q.count = reinterpret_cast<int *>(ws), q.index = reinterpret_cast<int *>(ws + plan.at_index), q.rows = reinterpret_cast<Row *>(ws + plan.at_rows);
    q.packed = reinterpret_cast<__nv_bfloat16 *>(ws + plan.at_packed);
    q.n = static_cast<int>(plan.n), q.dim = static_cast<int>(plan.dim), q.vocab = static_cast<int>(plan.vocab);
    q.each = static_cast<int>((plan.n + PRODUCT_SMS - 1) / PRODUCT_SMS);
    k_xent_rows<<<static_cast<unsigned>((plan.n + q.each - 1) / q.each), 256, 0, st>>>(q);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

// Tiles of rows to a band: a band of rows stays in the L2 while the columns pass.
int band_of(int64_t dim, int side) {
    const int64_t rows = (INT64_C(32) << 20) / (2 * dim);
    return rows < side ? 1 : rows / side > 1 << 20 ? 1 << 20 : static_cast<int>(rows / side);
}

int describe_rows(ProductMaps *maps, const Plan &plan, const void *hidden, int64_t hidden_stride, const char *ws, bool down) {
    CUtensorMap *const own = down ? &maps->b : &maps->a, *const packed = down ? &maps->b2 : &maps->a2;
    if (int rc = describe_operand(own, "hidden", false, down, hidden, plan.dim, plan.n, 1, hidden_stride * 2, 0)) return rc;
    return describe_operand(packed, "the workspace", false, down, ws + plan.at_packed, plan.dim, up(plan.n, K_STEP), 1, plan.dim * 2, 0);
}

template <template <bool> class Task, typename Params>
int start_either(bool pairs, const ProductMaps &maps, const Params &p, int64_t m, int64_t n, int64_t shares, cudaStream_t st) {
    const int side = pairs ? 256 : 128;
    const int64_t tiles = tiles_of(m, side) * tiles_of(n, side) * shares;
    return pairs ? start_product<Task<true>>(maps, p, tiles, st) : start_product<Task<false>>(maps, p, tiles, st);
}

}  // namespace

int ktd::xent_given_up(unsigned long long *count) {
    KT_CUDA(cudaMemcpyFromSymbol(count, g_waits_given_up, sizeof(*count)));
    return KT_OK;
}

extern "C" {

int64_t kt_xent_workspace(int64_t rows, int64_t dim, int64_t vocab, int backward) {
    if (rows < 1 || rows > MAX_ROWS || dim < 1 || dim > MAX_DIM || vocab < 1 || vocab > MAX_VOCAB) return 0;
    return Plan(rows, dim, vocab, backward != 0).bytes + 1024;
}

int kt_xent_forward(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, const int64_t *targets, float *loss, float *lse, void *workspace,
                    int64_t workspace_bytes, int64_t rows, int64_t dim, int64_t vocab, int dtype, float scale, void *stream) {
    if (int rc = check_common(rows, dim, vocab, dtype, scale)) return rc;
    if (rows == 0) return KT_OK;
    if (int rc = check_matrix("hidden", hidden, hidden_stride, rows, dim)) return rc;
    if (int rc = check_matrix("weight", weight, weight_stride, vocab, dim)) return rc;
    if (int rc = check_vector("targets", targets, 8)) return rc;
    if (int rc = check_vector("loss", loss, 4)) return rc;
    if (int rc = check_vector("lse", lse, 4)) return rc;
    const Plan plan(rows, dim, vocab, false);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.bytes + 1024)) return rc;
    char *const ws = reinterpret_cast<char *>(up(reinterpret_cast<intptr_t>(workspace), 1024));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProductMaps maps{};
    if (int rc = describe_rows(&maps, plan, hidden, hidden_stride, ws, false)) return rc;
    if (int rc = describe_operand(&maps.b, "weight", false, false, weight, dim, vocab, 1, weight_stride * 2, 0)) return rc;
    RowsParams q{};
    q.targets = targets, q.hidden = static_cast<const __nv_bfloat16 *>(hidden), q.hidden_stride = hidden_stride, q.loss_out = loss, q.lse_out = lse, q.scale = scale;
    if (int rc = start_rows(q, plan, ws, st)) return rc;
    const int side = plan.pairs_logits ? 256 : 128;
    LogitsParams p{};
    p.count = q.count, p.rows = q.rows, p.parts = reinterpret_cast<float2 *>(ws + plan.at_parts), p.at_target = reinterpret_cast<float *>(ws + plan.at_target);
    p.n = q.n, p.vocab = q.vocab, p.steps = static_cast<int>((dim + K_STEP - 1) / K_STEP), p.from = 0, p.past = q.vocab, p.band = band_of(dim, side), p.scale_log2 = scale * LOG2E;
    if (int rc = start_either<LossTask>(plan.pairs_logits, maps, p, rows, vocab, 1, st)) return rc;
    KT_CUDA(launch_behind(k_xent_join, 1, dim3(static_cast<unsigned>((rows + 7) / 8)), dim3(256), 0, st, static_cast<const int *>(q.count), static_cast<const int *>(q.index), static_cast<const Row *>(q.rows),
                          static_cast<const float2 *>(p.parts), static_cast<const float *>(p.at_target), q.n, static_cast<int>(tiles_of(vocab, side)), loss, lse));
    return KT_OK;
}

int kt_xent_backward(const float *dloss, const float *dlse, const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, const int64_t *targets, const float *lse,
                     void *dhidden, int64_t dhidden_stride, void *dweight, int64_t dweight_stride, void *workspace, int64_t workspace_bytes, int64_t rows, int64_t dim, int64_t vocab,
                     int dtype, float scale, void *stream) {
    if (int rc = check_common(rows, dim, vocab, dtype, scale)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dweight != nullptr)
        if (int rc = check_matrix("dweight", dweight, dweight_stride, vocab, dim)) return rc;
    if (rows == 0) {
        if (dweight != nullptr) KT_CUDA(cudaMemset2DAsync(dweight, static_cast<size_t>(vocab > 1 ? dweight_stride : dim) * 2, 0, static_cast<size_t>(dim) * 2, static_cast<size_t>(vocab), st));
        return KT_OK;
    }
    if (dhidden == nullptr && dweight == nullptr) return fail(KT_ERR_INVALID, "dhidden and dweight are both NULL");
    if (int rc = check_matrix("hidden", hidden, hidden_stride, rows, dim)) return rc;
    if (int rc = check_matrix("weight", weight, weight_stride, vocab, dim)) return rc;
    if (dhidden != nullptr)
        if (int rc = check_matrix("dhidden", dhidden, dhidden_stride, rows, dim)) return rc;
    if (int rc = check_vector("targets", targets, 8)) return rc;
    if (int rc = check_vector("dloss", dloss, 4)) return rc;
    if (int rc = check_vector("dlse", dlse, 4, true)) return rc;
    if (int rc = check_vector("lse", lse, 4)) return rc;
    const Plan plan(rows, dim, vocab, true);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.bytes + 1024)) return rc;
    char *const ws = reinterpret_cast<char *>(up(reinterpret_cast<intptr_t>(workspace), 1024));
    float *const sums = reinterpret_cast<float *>(ws + plan.at_sums);
    const bool direct = plan.pieces == 1 && plan.shares == 1;
    const int64_t p_rows = up(rows, TILE), pitch = plan.piece * 2;

    ProductMaps logits{}, to_hidden{}, to_weight{};
    if (int rc = describe_rows(&logits, plan, hidden, hidden_stride, ws, false)) return rc;
    if (int rc = describe_operand(&logits.b, "weight", false, false, weight, dim, vocab, 1, weight_stride * 2, 0)) return rc;
    if (int rc = describe_matrix(&logits.out, "the workspace", CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0, 64, 32)) return rc;
    if (dhidden != nullptr) {
        if (int rc = describe_operand(&to_hidden.a, "the workspace", false, false, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0)) return rc;
        if (!direct)
            if (int rc = describe_matrix(&to_hidden.out, "the workspace", CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, sums, dim, rows, plan.shares, dim * 4, rows * dim * 4, 32, 32)) return rc;
    }
    if (dweight != nullptr) {
        if (int rc = describe_operand(&to_weight.a, "the workspace", false, true, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0)) return rc;
        if (int rc = describe_rows(&to_weight, plan, hidden, hidden_stride, ws, true)) return rc;
        if (int rc = describe_matrix(&to_weight.out, "dweight", CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dweight, dim, vocab, 1, dweight_stride * 2, 0, 64, 32)) return rc;
    }

    RowsParams q{};
    q.targets = targets, q.hidden = static_cast<const __nv_bfloat16 *>(hidden), q.hidden_stride = hidden_stride, q.scale = scale;
    q.dloss = dloss, q.dlse = dlse, q.lse = lse, q.dhidden = static_cast<__nv_bfloat16 *>(dhidden), q.dhidden_stride = dhidden_stride;
    if (int rc = start_rows(q, plan, ws, st)) return rc;
    for (int64_t i = 0; i < plan.pieces; ++i) {
        const int64_t from = i * plan.piece, past = from + plan.piece < vocab ? from + plan.piece : vocab;
        LogitsParams p{};
        p.count = q.count, p.rows = q.rows, p.n = q.n, p.vocab = q.vocab, p.steps = static_cast<int>((dim + K_STEP - 1) / K_STEP);
        p.from = static_cast<int>(from), p.past = static_cast<int>(past), p.band = band_of(dim, plan.pairs_logits ? 256 : 128), p.scale_log2 = scale * LOG2E;
        if (int rc = start_either<GradTask>(plan.pairs_logits, logits, p, rows, past - from, 1, st)) return rc;
        if (dhidden != nullptr) {
            if (int rc = describe_operand(&to_hidden.b, "weight", false, true, static_cast<const __nv_bfloat16 *>(weight) + from * weight_stride, dim, past - from, 1, weight_stride * 2, 0)) return rc;
            HiddenParams h{};
            const int64_t steps = (past - from + K_STEP - 1) / K_STEP;
            h.count = q.count, h.index = q.index, h.to = direct ? q.dhidden : nullptr, h.to_stride = dhidden_stride;
            h.tiles_n = static_cast<int>(tiles_of(dim, plan.pairs_hidden ? 256 : 128)), h.band = 8, h.dim = q.dim;
            h.shares = static_cast<int>(plan.shares), h.steps = static_cast<int>(steps), h.add = i > 0;
            if (int rc = start_either<HiddenTask>(plan.pairs_hidden, to_hidden, h, rows, dim, plan.shares, st)) return rc;
        }
        if (dweight != nullptr) {
            const int side = plan.pairs_weight ? 256 : 128;
            WeightParams w{};
            w.count = q.count, w.n = q.n, w.tiles_m = static_cast<int>(tiles_of(past - from, side)), w.tiles_n = static_cast<int>(tiles_of(dim, side)), w.band = 8, w.vocab = static_cast<int>(past), w.dim = q.dim,
            w.from = static_cast<int>(from);
            if (int rc = start_either<WeightTask>(plan.pairs_weight, to_weight, w, past - from, dim, 1, st)) return rc;
        }
    }
    if (dhidden != nullptr && !direct) {
        const int64_t blocks = (rows * (dim / 8) + 255) / 256;
        KT_CUDA(launch_behind(k_xent_dhidden, 1, dim3(static_cast<unsigned>(blocks < 8 * PRODUCT_SMS ? blocks : 8 * PRODUCT_SMS)), dim3(256), 0, st, static_cast<const int *>(q.count),
                              static_cast<const int *>(q.index), static_cast<const float *>(sums), static_cast<int>(plan.shares), rows * dim, q.dim, q.dhidden, dhidden_stride));
    }
    return KT_OK;
}

}  // extern "C"
