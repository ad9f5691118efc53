// kt_xent.cu -- softmax cross entropy of hidden rows against the weights of a vocabulary, with its gradient, without
// keeping the logits.  Contracts: include/kaitian.h.
//
// With logits l_iv = scale h_i . w_v and lse_i = log sum_v exp(l_iv):
//   forward    loss_i = lse_i - l_{i, t_i}
//   backward   P_iv = scale ((g_i + z_i) exp(l_iv - lse_i) - g_i [v = t_i])  for dloss g and dlse z,
//              dh = P W,  dW = P^T h
// P is held as Q_iv = P_iv / u_i with a unit u_i = scale g_i of each row, so that a target's entry is near -1: in bf16 that of
// P itself would be off by up to 2^-9 in the same direction in all rows of equal g (a mean's 1 / n), which with a large
// vocabulary is nearly all there is (0.3 % in both gradients, where Q gives 0.17 %, what their own rounding is).  dh_i = u_i (Q W)_i
// and, where all u_i are the same, dW = u Q^T h; else hidden rows are multiplied by u_i before.
// Three kinds of products (kt_product.cuh):
//   loss   a tile of logits becomes a maximum, a sum of exponentials and perhaps the target's logit of each row
//   grad   the logits are formed again, and leave the chip as Q in bf16, a piece of the vocabulary at a time (the second
//          products of the tensor cores take 16-bit operands; bf16 because Q spans the range of probabilities)
//   back   dh and dW from the piece.  dW of the piece's rows is whole; dh is summed over the pieces in fp32.
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
    float all, target_part;                     // (g + z) / unit, g / unit (without scale)
};
// What the rows have in common, at the start of the workspace.
struct Common {
    int count;                                  // rows that count
    int one_unit;                               // whether all have the same unit
    float unit;
};
constexpr int PAST_VOCAB = 0x7FFFFFFF;

__device__ __forceinline__ int round_to(int x, int m) { return (x + m - 1) / m * m; }

// ------------------------------------------------------------------------------ rows that count
struct RowsParams {
    const int64_t *targets;
    const __nv_bfloat16 *hidden;
    int64_t hidden_stride;
    __nv_bfloat16 *packed;                      // counted rows of hidden, where some do not count
    __nv_bfloat16 *scaled;                      // those times their units, where these differ (backward)
    Common *common;
    int *index;                                 // index[i]: the row that is the i-th to count
    Row *rows;
    float *units;
    const float *dloss, *dlse, *lse;            // backward
    float *loss_out, *lse_out;                  // forward
    __nv_bfloat16 *dhidden;
    int64_t dhidden_stride;
    int n, dim, vocab, each;                    // each: rows to a CTA
    float scale;
};

// A row's unit without the scale: g, or g + z where that is far more.
__device__ __forceinline__ float unit_of(float g, float z) { return fabsf(g) * 256.0f < fabsf(g + z) ? g + z : g; }      // (NaN: NaN)

__device__ __forceinline__ uint32_t times(uint32_t two, float by) {
    return pack_bf16(__uint_as_float(two << 16) * by, __uint_as_float(two & 0xFFFF0000u) * by);
}

// Every CTA goes over all targets to find out where its own rows begin (and, backward, over the gradients: whether the rows have
// one unit), so no CTA waits for another.  Latency: 4 us for 200 rows, 12 where 1600 of 4096 rows of 2048 are left out.
__global__ void __launch_bounds__(256) k_xent_rows(const RowsParams p) {
    __shared__ int sums[8], sums_before[8], place[256];
    __shared__ unsigned least[8], most[8];
    __shared__ float unit_at[256];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    let_next_begin();
    const int begin = min(p.n, static_cast<int>(blockIdx.x) * p.each), end = min(p.n, begin + p.each);
    const bool back = p.lse != nullptr;
    int before = 0, all = 0;
    unsigned low = 0xFFFFFFFFu, high = 0;       // of the units' bits
    for (int i0 = tid; i0 < p.n; i0 += 8 * 256) {       // (all asked for at once, whether they count or not)
        int64_t target[8];
        float g[8], z[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) target[u] = i0 + u * 256 < p.n ? p.targets[i0 + u * 256] : -1;
        if (back) {
#pragma unroll
            for (int u = 0; u < 8; ++u) g[u] = i0 + u * 256 < p.n ? p.dloss[i0 + u * 256] : 0.0f, z[u] = p.dlse != nullptr && i0 + u * 256 < p.n ? p.dlse[i0 + u * 256] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const bool counts = target[u] >= 0;
            all += counts, before += counts && i0 + u * 256 < begin;
            if (back && counts) {
                const unsigned bits = __float_as_uint(p.scale * unit_of(target[u] < p.vocab ? g[u] : __int_as_float(0x7FFFFFFF), z[u]));
                low = min(low, bits), high = max(high, bits);
            }
        }
    }
    all = __reduce_add_sync(0xFFFFFFFFu, all), before = __reduce_add_sync(0xFFFFFFFFu, before);
    low = __reduce_min_sync(0xFFFFFFFFu, low), high = __reduce_max_sync(0xFFFFFFFFu, high);
    if (lane == 0) sums[warp] = all, sums_before[warp] = before, least[warp] = low, most[warp] = high;
    __syncthreads();
    all = before = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) all += sums[w], before += sums_before[w], low = min(low, least[w]), high = max(high, most[w]);
    const bool copy = all < p.n, one_unit = low >= high, scale_rows = back && !one_unit;       // (no row that counts: one unit)
    const int pieces = p.dim / 8;
    if (blockIdx.x == 0) {
        if (tid == 0) *p.common = {all, one_unit, __uint_as_float(high)};
        // a stage of the reduction over rows may read past the last: zeros there
        for (int64_t i = static_cast<int64_t>(all) * pieces + tid; i < static_cast<int64_t>(round_to(all, K_STEP)) * pieces; i += 256) {
            if (copy) reinterpret_cast<uint4 *>(p.packed)[i] = make_uint4(0, 0, 0, 0);
            if (scale_rows) reinterpret_cast<uint4 *>(p.scaled)[i] = make_uint4(0, 0, 0, 0);
        }
    }
    for (int base = begin; base < end; base += 256) {
        const int i = base + tid;
        const int64_t target = i < end ? p.targets[i] : -1;
        const float own_g = back && i < end ? p.dloss[i] : 0.0f, own_z = back && p.dlse != nullptr && i < end ? p.dlse[i] : 0.0f, own_lse = back && i < end ? p.lse[i] : 0.0f;
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
            if (back) {
                const float g = known ? own_g : __int_as_float(0x7FFFFFFF), z = own_z, u = unit_of(g, z);
                row.lse2 = own_lse * LOG2E;
                if (u != 0.0f) row.all = (g + z) / u, row.target_part = g / u;       // (exactly 1 where the unit is g)
                p.units[at] = unit_at[tid] = u * p.scale;
            }
            p.rows[at] = row, p.index[at] = i;
        } else if (i < end && p.loss_out != nullptr) {
            p.loss_out[i] = 0.0f, p.lse_out[i] = 0.0f;
        }
        if (!copy && !scale_rows) continue;
        __syncthreads();
        for (int r = warp; r < min(256, end - base); r += 8) {
            const int to = place[r];
            if (to >= 0) {
                const uint4 *from = reinterpret_cast<const uint4 *>(p.hidden + (base + r) * p.hidden_stride);
                uint4 *const row = reinterpret_cast<uint4 *>(p.packed + static_cast<int64_t>(to) * p.dim), *const scaled = reinterpret_cast<uint4 *>(p.scaled + static_cast<int64_t>(to) * p.dim);
                const float by = unit_at[r];
#pragma unroll 8
                for (int c = lane; c < pieces; c += 32) {
                    const uint4 v = from[c];
                    if (copy) row[c] = v;
                    if (scale_rows) scaled[c] = make_uint4(times(v.x, by), times(v.y, by), times(v.z, by), times(v.w, by));
                }
            } else if (p.dhidden != nullptr) {
                uint4 *const row = reinterpret_cast<uint4 *>(p.dhidden + (base + r) * p.dhidden_stride);
                for (int c = lane; c < pieces; c += 32) row[c] = make_uint4(0, 0, 0, 0);
            }
        }
    }
}

// ------------------------------------------------------------------------------------ products
// Operands, each read in up to two or three ways, and results.
struct LogitsMaps {
    CUtensorMap hidden, packed, weight, p;      // rows as they are, or those that count
};
struct BackMaps {
    CUtensorMap p, p_down, weight, hidden, packed, scaled, dweight, sums;
};

// Rows that a box of hidden rows, or of P, brings: no more than there are.  (The rest of a tile holds what was there before;
// its results are nobody's.)
__host__ __device__ inline int rows_of_box(int64_t n) { return n < TILE ? static_cast<int>((n + 7) / 8 * 8) : TILE; }

// The order of tiles: bands of up to `band` tiles of rows, in a band column after column, so that the tiles
// in work at one time share rows and columns that the L2 holds.
__device__ __forceinline__ void in_bands(int i, int tiles_m, int tiles_n, int band, int *m, int *n) {
    band = min(band, tiles_m);
    const int per_band = band * tiles_n, b = i / per_band, in = i - b * per_band, high = min(band, tiles_m - b * band);
    *n = in / high;
    *m = b * band + in - *n * high;
}

struct LogitsParams {
    const Common *common;
    const int *index;
    const Row *rows;
    const int64_t *targets;                     // where nothing was left out, because one tile holds all rows: instead of the three
    float2 *parts;                              // [half tiles of columns][n]: maximum (units of log 2) and sum
    float *at_target;                           // the target's logit (units of log 2)
    int n, vocab, steps, from, past, band;      // columns from ... past of the vocabulary
    float scale_log2;
    __device__ __forceinline__ int counted() const { return targets != nullptr ? n : common->count; }
    __device__ __forceinline__ Row row(int i) const {
        if (targets == nullptr) return rows[i];
        const int64_t t = targets[i];
        return {t < 0 ? -1 : t < vocab ? static_cast<int>(t) : PAST_VOCAB, 0.0f, 0.0f, 0.0f};
    }
};

template <bool PAIR_>
struct LogitsTask {
    using Params = LogitsParams;
    using Maps = LogitsMaps;
    static constexpr bool PAIR = PAIR_, HALF = false;
    static constexpr int SIDE = PAIR ? 256 : 128;
    struct Cut {
        int counted, n, from, steps, tiles_m, tiles_n, band, worker, workers;
        __device__ Cut(const Params &p, int worker_, int workers_) : counted(p.counted()), n(p.n), from(p.from), steps(p.steps), band(p.band), worker(worker_), workers(workers_) {
            tiles_m = (counted + SIDE - 1) / SIDE, tiles_n = (p.past - p.from + SIDE - 1) / SIDE;
        }
        __device__ int count() const { return (tiles_m * tiles_n - worker + workers - 1) / workers; }
        __device__ Tile tile(int i) const {
            int m, n;
            in_bands(worker + i * workers, tiles_m, tiles_n, band, &m, &n);
            return {m * SIDE, from + n * SIDE, 0, 0, steps, 0, 0};
        }
    };
    __device__ static bool a_down(const Tile &) { return false; }
    __device__ static bool b_down(const Tile &) { return false; }
    __device__ static const CUtensorMap *map_a(const Maps &maps, const Cut &c, const Tile &) { return c.counted < c.n ? &maps.packed : &maps.hidden; }
    __device__ static const CUtensorMap *map_b(const Maps &maps, const Cut &, const Tile &) { return &maps.weight; }
    __device__ static int rows_a(const Cut &c, const Tile &) { return rows_of_box(c.n); }
};

// A thread has half of a row of a tile: maximum and sum of exponentials (base 2) in one pass, 32 columns at a time.  With 512
// elements of reduction and less this, not the product, is what a tile takes (4.2 us of which the tensor cores are busy 59 %: 8192 rows, 512,
// 32000: 225 us, floor 161).  No rate bounds it (exponentials' unit 32 % busy, instructions in 35 % of the cycles): most of what a warp waits for is the instruction before, in
// the chain of maximum, rescaling, exponentials and sum to every 32 columns, with two warps to a scheduler.  With 4096 and up the tensor cores at the power limit (8192 rows, 65536: 2762 to 3054 us as the clocks go).
template <bool PAIR_>
struct LossTask : LogitsTask<PAIR_> {
    using Base = LogitsTask<PAIR_>;
    __device__ static void finish(const LogitsParams &p, const LogitsMaps &, const typename Base::Cut &cut, const Tile &, Part &part) {
        const bool counts = part.row < cut.counted;
        const int target = counts ? p.row(part.row).target : -1;
        float top = -INFINITY, sum = 0.0f;
        over_columns<Base::SIDE / 2>(part, [&](int v0, auto half, uint32_t (&r)[32]) {
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
        if (counts) p.parts[static_cast<int64_t>(part.col / (Base::SIDE / 2)) * p.n + part.row] = make_float2(top, sum);
    }
};

// 64 columns of a row, as 16-bit values, through the store to a matrix.
template <typename F>
__device__ __forceinline__ void pack_row(const Part &part, int half, F value) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint4 v;
        v.x = pack_bf16(value(u * 8), value(u * 8 + 1)), v.y = pack_bf16(value(u * 8 + 2), value(u * 8 + 3));
        v.z = pack_bf16(value(u * 8 + 4), value(u * 8 + 5)), v.w = pack_bf16(value(u * 8 + 6), value(u * 8 + 7));
        *part.piece(half * 4 + u) = v;
    }
}

// The same pass with the row's lse: Q, through the store in shared memory (4096 x 1024 on 50257: 280 us for 422 GFLOP, 412 MB of
// Q written beside).
template <bool PAIR_>
struct GradTask : LogitsTask<PAIR_> {
    using Base = LogitsTask<PAIR_>;
    __device__ static void finish(const LogitsParams &p, const LogitsMaps &maps, const typename Base::Cut &cut, const Tile &, Part &part) {
        const int count = cut.counted;
        if (part.warp_row >= round_to(count, TILE)) return;
        const bool counts = part.row < count;
        const Row row = counts ? p.rows[part.row] : Row{-1, 0.0f, 0.0f, 0.0f};
        over_columns<Base::SIDE / 2>(part, [&](int v0, auto half, uint32_t (&r)[32]) {
            if (v0 - half * 32 >= p.past) return;
            if (half == 0) part.store_next();
            const int d = row.target - v0, left = p.past - v0;
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 y = fma2(pair_of(r, e), both(p.scale_log2), both(-row.lse2));
                const float2 g = mul2(make_float2(exp2_fast(y.x), exp2_fast(y.y)), both(row.all));
                x[e] = g.x, x[e + 1] = g.y;
            }
            if (static_cast<unsigned>(d) < 32u)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e == d) x[e] -= row.target_part;
            if (!counts || left < 32)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (!counts || e >= left) x[e] = 0.0f;
            pack_row(part, half, [&](int e) { return x[e]; });
            if (half == 1) part.send(&maps.p, v0 - 32 - p.from, part.warp_row, 0);
        });
    }
};

// Both products of a piece of P in one launch, since neither waits for the other: first the tiles of dh, reduced over the
// piece's columns or a share of them, then those of dW, reduced over the counted rows.  A tile of dh takes long where the piece is wide,
// and there are few of them: workers that do one less of them do more of dW's.
struct BackParams {
    const Common *common;
    const int *index;
    const float *units;
    __nv_bfloat16 *to;                          // dh where a tile has all of it; else NULL, and its shares are added up in fp32
    int64_t to_stride;
    int n, dim, from, past;                     // from ... past: columns of the vocabulary
    int tiles_n, tiles_w, shares, steps, add;   // tiles across dim and (dW) across the piece; shares of the piece's stages; whether to add
    int hidden;                                 // whether dh is wanted
};
template <bool PAIR_>
struct BackTask {
    using Params = BackParams;
    using Maps = BackMaps;
    static constexpr bool PAIR = PAIR_, HALF = false;
    static constexpr int SIDE = PAIR ? 256 : 128, BAND = 8;
    static constexpr int FINISH = 2;            // stages' time that a tile's end takes
    struct Cut {
        int counted, n, one_unit;
        float unit;
        int worker, workers, steps, shares, tiles_m, tiles_n, tiles_w, weight_steps;
        int mine, early, late;                  // tiles of dh; of dW while others are at a tile of dh more; and after
        int skip, others, meanwhile;            // workers with a tile of dh more, those without, what the latter do before the rest
        __device__ Cut(const Params &p, int worker_, int workers_) : counted(p.common->count), n(p.n), one_unit(p.common->one_unit), unit(p.common->unit), worker(worker_), workers(workers_), steps(p.steps), shares(p.shares), tiles_n(p.tiles_n), tiles_w(p.tiles_w) {
            tiles_m = (counted + SIDE - 1) / SIDE, weight_steps = (counted + K_STEP - 1) / K_STEP;
            const int hidden = p.hidden ? tiles_m * tiles_n * shares : 0, weight = tiles_w * tiles_n, each = hidden / workers;
            skip = hidden - each * workers, others = workers - skip;
            const int more = skip == 0 ? 0 : min((steps / shares + FINISH) / (weight_steps + FINISH), (weight + others - 1) / others);
            meanwhile = min(weight, others * more);
            mine = each + (worker < skip ? 1 : 0);
            early = worker < skip ? 0 : (meanwhile - (worker - skip) + others - 1) / others;
            late = (weight - meanwhile + worker) / workers;
        }
        __device__ int count() const { return mine + early + late; }
        __device__ Tile tile(int i) const {
            int row, col;
            if (i < mine) {
                const int at = worker + i * workers, share = at % shares;
                const int begin = steps * share / shares, end = steps * (share + 1) / shares;      // (32768 stages at most, 16 to a share)
                in_bands(at / shares, tiles_m, tiles_n, BAND, &row, &col);
                return {row * SIDE, col * SIDE, 0, begin * K_STEP, end - begin, 0, share};
            }
            i -= mine;
            in_bands(i < early ? worker - skip + i * others : meanwhile + (workers - 1 - worker) + (i - early) * workers, tiles_w, tiles_n, BAND, &row, &col);
            return {row * SIDE, col * SIDE, 0, 0, weight_steps, 1, 0};
        }
    };
    __device__ static bool a_down(const Tile &t) { return t.kind == 1; }
    __device__ static bool b_down(const Tile &) { return true; }
    __device__ static const CUtensorMap *map_a(const Maps &maps, const Cut &, const Tile &t) { return t.kind == 0 ? &maps.p : &maps.p_down; }
    __device__ static int rows_a(const Cut &c, const Tile &) { return rows_of_box(c.n); }
    __device__ static const CUtensorMap *map_b(const Maps &maps, const Cut &c, const Tile &t) { return t.kind == 0 ? &maps.weight : !c.one_unit ? &maps.scaled : c.counted < c.n ? &maps.packed : &maps.hidden; }
    __device__ static void finish(const Params &p, const Maps &maps, const Cut &cut, const Tile &t, Part &part) {
        const int count = cut.counted;
        const bool weight = t.kind == 1;
        if (weight ? p.from + part.warp_row >= p.past : part.warp_row >= count) return;
        const float unit = !weight ? (part.row < count ? p.units[part.row] : 0.0f) : cut.one_unit ? cut.unit : 1.0f;
        __nv_bfloat16 *const row = !weight && p.to != nullptr && part.row < count ? p.to + p.index[part.row] * p.to_stride : nullptr;
        over_columns<SIDE / 2>(part, [&](int c0, auto half, uint32_t (&r)[32]) {
            if (weight) {
                if (c0 - half * 32 >= p.dim) return;
                if (half == 0) part.store_next();
                pack_row(part, half, [&](int e) { return __uint_as_float(r[e]) * unit; });
                if (half == 1) part.send(&maps.dweight, c0 - 32, p.from + part.warp_row, 0);
            } else if (p.to == nullptr) {
                if (c0 >= p.dim) return;
                part.store_next();
#pragma unroll
                for (int u = 0; u < 8; ++u) *part.piece(u) = make_uint4(r[u * 4], r[u * 4 + 1], r[u * 4 + 2], r[u * 4 + 3]);       // (units come with the shares' sum)
                part.send(&maps.sums, c0, part.warp_row, t.share, p.add != 0);
            } else if (row != nullptr) {
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if (c0 + e < p.dim) {
                        uint4 v;
                        v.x = pack_bf16(mul2(pair_of(r, e), both(unit))), v.y = pack_bf16(mul2(pair_of(r, e + 2), both(unit)));
                        v.z = pack_bf16(mul2(pair_of(r, e + 4), both(unit))), v.w = pack_bf16(mul2(pair_of(r, e + 6), both(unit)));
                        *reinterpret_cast<uint4 *>(row + c0 + e) = v;
                    }
            }
        });
    }
};

// ------------------------------------------------------------------------------------- ends
// The parts of a row joined; 8 rows to a CTA, 32 threads to a row, eight parts on their way to a thread at a time.
__global__ void __launch_bounds__(256) k_xent_join(const LogitsParams p, int tiles, float *loss, float *lse) {
    __shared__ float2 of_warp[8][8];
    let_next_begin();
    after_previous();
    const int tid = threadIdx.x, r = tid % 8, row = blockIdx.x * 8 + r;
    const bool there = row < p.counted();
    float top = -INFINITY, sum = 0.0f;
    auto join = [&](float2 x) {
        const float high = fmaxf(top, x.x), zero = high == -INFINITY ? 0.0f : high;
        sum = sum * exp2_fast(top - zero) + x.y * exp2_fast(x.x - zero);
        top = high;
    };
    const Row mine = there ? p.row(row) : Row{-1, 0.0f, 0.0f, 0.0f};
    const float at = there ? p.at_target[row] : 0.0f;
    const int to = there && p.index != nullptr ? p.index[row] : row;
    if (there)
        for (int i0 = tid / 8; i0 < tiles; i0 += 8 * 32) {
            float2 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = i0 + u * 32 < tiles ? p.parts[static_cast<int64_t>(i0 + u * 32) * p.n + row] : make_float2(-INFINITY, 0.0f);
            float high = -INFINITY, part = 0.0f;
#pragma unroll
            for (int u = 0; u < 8; ++u) high = fmaxf(high, x[u].x);
            const float zero = high == -INFINITY ? 0.0f : high;
#pragma unroll
            for (int u = 0; u < 8; ++u) part += x[u].y * exp2_fast(x[u].x - zero);
            join(make_float2(high, part));
        }
#pragma unroll
    for (int far = 8; far < 32; far *= 2) join(make_float2(__shfl_xor_sync(0xFFFFFFFFu, top, far), __shfl_xor_sync(0xFFFFFFFFu, sum, far)));
    if (tid % 32 < 8) of_warp[tid / 32][r] = make_float2(top, sum);
    __syncthreads();
    if (tid >= 8 || !there) return;
    top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) join(of_warp[w][r]);
    const float high = log2f(sum);
    const bool counts = mine.target >= 0;       // (a row that does not count is among these where nothing was left out)
    lse[to] = counts ? (top + high) * LN2 : 0.0f;
    // the maximum and the target's logit first: they are close where the loss is small
    loss[to] = !counts ? 0.0f : mine.target == PAST_VOCAB ? __int_as_float(0x7FFFFFFF) : ((top - at) + high) * LN2;
}

// The shares of dh added up, in order, and given their rows' units.
__global__ void __launch_bounds__(256) k_xent_dhidden(const Common *common, const int *index, const float *units, const float *sums, int shares, int64_t share, int dim, __nv_bfloat16 *to, int64_t stride) {
    let_next_begin();
    after_previous();
    const uint32_t pieces = dim / 8, all = common->count, step = gridDim.x * 256, step_rows = step / pieces, step_pieces = step % pieces, first = blockIdx.x * 256 + threadIdx.x;
    uint32_t piece = first % pieces;
    for (uint32_t row = first / pieces; row < all; row += step_rows, piece += step_pieces) {
        if (piece >= pieces) {
            piece -= pieces;
            if (++row >= all) break;
        }
        const int c = piece * 8;
        const float *from = sums + static_cast<int64_t>(row) * dim + c;
        float4 a = *reinterpret_cast<const float4 *>(from), b = *reinterpret_cast<const float4 *>(from + 4);
#pragma unroll 4
        for (int s = 1; s < shares; ++s) {
            const float4 c0 = *reinterpret_cast<const float4 *>(from + s * share), c1 = *reinterpret_cast<const float4 *>(from + s * share + 4);
            a.x += c0.x, a.y += c0.y, a.z += c0.z, a.w += c0.w, b.x += c1.x, b.y += c1.y, b.z += c1.z, b.w += c1.w;
        }
        uint4 v;
        const float u = units[row];
        v.x = pack_bf16(a.x * u, a.y * u), v.y = pack_bf16(a.z * u, a.w * u), v.z = pack_bf16(b.x * u, b.y * u), v.w = pack_bf16(b.z * u, b.w * u);
        *reinterpret_cast<uint4 *>(to + index[row] * stride + c) = v;
    }
}

// ---------------------------------------------------------------------------------- host side
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
int64_t tiles_of(int64_t x, int side) { return (x + side - 1) / side; }

// Whether the logits' tiles are worked on by pairs of CTAs: where there are almost as many tiles of 256 x 256 as pairs, and not
// where half of a tile would be empty rows.  In us, one CTA to a tile and pairs:
//   forward, 200 x 512 on 8001 (32 tiles)       12.4  14.4        512 x 1024 on 8001 (64)     20.5  18.6
//   forward, 512 x 512 on 8001 (64)             16.5  16.5        200 x 512 on 32000 (125)    23.8  20.5
bool by_pairs(int64_t m, int64_t n) { return m > TILE && tiles_of(m, 256) * tiles_of(n, 256) >= 60; }

// The same for the products from P, which differ in length: by the stages of the reductions that a pair would have.  In us, one CTA to a tile
// and pairs (all kernels of the backward pass):
//   200 x 768 on 8001 (10 stages)     28.2  29.6        512 x 1024 on 8001 (27)     43.2  39.5        400 x 512 on 32000 (50)     74.3  66.8
//   512 x 512 on 8001 (13)            30.9  32.0        1000 x 512 on 8001 (27)     44.6  40.1        1000 x 768 on 8001 (41)     57.6  46.5
//   256 x 512 on 16000 (13)           32.3  38.3        200 x 4096 on 4001 (27)     55.3  51.0        200 x 1024 on 32000 (54)    80.4  78.8
//   200 x 2048 on 8001 (27)           48.7  45.4        512 x 512 on 16000 (27)     46.3  43.7        512 x 1024 on 32000 (108)    129   101
// Up to 300 rows with up to 1024 elements pairs are the slower ones up to some 43 stages, since dW's tiles have 4 or 5 stages each and wait for their ends, which
// the rule does not look at: 200 x 512 on 32000 (27) 50.2 and 56.4, 200 x 1024 on 16000 (27) 46.8 and 48.5, 300 x 768 on 16000 (33) 48.2 and 50.5,
// 200 x 768 on 32000 (40) 64.0 and 66.2, 300 x 512 on 32000 (43) 64.5 and 69.5.
constexpr int64_t PAIR_STAGES = 24;

constexpr int64_t PIECE_BYTES = INT64_C(512) << 20;        // of P, at most

// Where everything lies in the workspace, and how the work is cut: from the sizes alone.
struct Plan {
    int64_t n, dim, vocab;
    bool backward;
    int64_t piece, pieces, shares;              // columns of the vocabulary to a piece; shares of dh's reduction
    bool pairs_logits, pairs_back;
    int64_t at_index, at_rows, at_units, at_packed, at_scaled, at_parts, at_target, at_p, at_sums, bytes;
    Plan(int64_t rows, int64_t dims, int64_t words, bool back) : n(rows), dim(dims), vocab(words), backward(back) {
        int64_t at = 0;
        auto take = [&](int64_t size) {
            const int64_t here = at;
            at += up(size, 1024);
            return here;
        };
        take(sizeof(Common));
        at_index = take(4 * n), at_rows = take(static_cast<int64_t>(sizeof(Row)) * n);
        at_units = take(backward ? 4 * n : 0);
        at_packed = take(2 * up(n, K_STEP) * dim), at_scaled = take(backward ? 2 * up(n, K_STEP) * dim : 0);
        const int64_t room = PIECE_BYTES / (2 * up(n, TILE)) / 256 * 256, most = room < 256 ? 256 : room;
        pieces = backward ? tiles_of(vocab, static_cast<int>(most)) : 1;
        piece = backward ? up((vocab + pieces - 1) / pieces, 256) : vocab;
        pieces = (vocab + piece - 1) / piece;
        pairs_logits = by_pairs(n, piece);
        const int64_t steps = (piece + K_STEP - 1) / K_STEP, over_rows = (n + K_STEP - 1) / K_STEP;
        auto stages = [&](int side, int64_t workers) { return tiles_of(dim, side) * (tiles_of(n, side) * steps + tiles_of(piece, side) * over_rows) / workers; };
        pairs_back = n > TILE && stages(256, PRODUCT_SMS / 2) >= PAIR_STAGES;
        // dh: shares of the piece such that a tile takes no longer than all work on all workers, but 16 stages at least (with 8: 38.4 us
        // instead of 33.5 for 200 x 768 on 8001, with 32 34.9)
        const int64_t mean = pairs_back ? stages(256, PRODUCT_SMS / 2) : stages(128, PRODUCT_SMS), longest = mean < 16 ? 16 : mean;
        shares = (steps + longest - 1) / longest;
        at_parts = take(backward ? 0 : 8 * n * 2 * tiles_of(vocab, pairs_logits ? 256 : 128)), at_target = take(backward ? 0 : 4 * n);
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
    q.common = reinterpret_cast<Common *>(ws), q.units = reinterpret_cast<float *>(ws + plan.at_units), q.index = reinterpret_cast<int *>(ws + plan.at_index), q.rows = reinterpret_cast<Row *>(ws + plan.at_rows);
    q.packed = reinterpret_cast<__nv_bfloat16 *>(ws + plan.at_packed), q.scaled = reinterpret_cast<__nv_bfloat16 *>(ws + plan.at_scaled);
    q.n = static_cast<int>(plan.n), q.dim = static_cast<int>(plan.dim), q.vocab = static_cast<int>(plan.vocab);
    q.each = static_cast<int>((plan.n + 4 * PRODUCT_SMS - 1) / (4 * PRODUCT_SMS));      // four CTAs to an SM
    if (q.each < 8) q.each = 8;                 // a row to a warp
    k_xent_rows<<<static_cast<unsigned>((plan.n + q.each - 1) / q.each), 256, 0, st>>>(q);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

// Tiles of rows to a band: a band of rows stays in the L2 while the columns pass.
int band_of(int64_t dim, int side) {
    const int64_t rows = (INT64_C(32) << 20) / (2 * dim);
    return rows < side ? 1 : rows / side > 1 << 20 ? 1 << 20 : static_cast<int>(rows / side);
}

// The counted rows: hidden itself where all count, and where they have been copied to.
int describe_rows(CUtensorMap *own, CUtensorMap *packed, const Plan &plan, const void *hidden, int64_t hidden_stride, const char *ws, bool down) {
    if (int rc = describe_operand(own, "hidden", false, down, hidden, plan.dim, plan.n, 1, hidden_stride * 2, 0, rows_of_box(plan.n))) return rc;
    return describe_operand(packed, "the workspace", false, down, ws + plan.at_packed, plan.dim, up(plan.n, K_STEP), 1, plan.dim * 2, 0, rows_of_box(plan.n));
}

template <template <bool> class Task, typename Params>
int start_either(bool pairs, const typename Task<false>::Maps &maps, const Params &p, int64_t tiles, cudaStream_t st, bool behind = true) {
    return pairs ? start_product<Task<true>>(maps, p, tiles, st, behind) : start_product<Task<false>>(maps, p, tiles, st, behind);
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
    LogitsMaps maps{};
    if (int rc = describe_rows(&maps.hidden, &maps.packed, plan, hidden, hidden_stride, ws, false)) return rc;
    if (int rc = describe_operand(&maps.weight, "weight", false, false, weight, dim, vocab, 1, weight_stride * 2, 0)) return rc;
    LogitsParams p{};
    p.parts = reinterpret_cast<float2 *>(ws + plan.at_parts), p.at_target = reinterpret_cast<float *>(ws + plan.at_target);
    const int side = plan.pairs_logits ? 256 : 128;
    p.n = static_cast<int>(rows), p.vocab = p.past = static_cast<int>(vocab), p.steps = static_cast<int>((dim + K_STEP - 1) / K_STEP), p.band = band_of(dim, side), p.scale_log2 = scale * LOG2E;
    const bool leave_out = rows > side;         // one tile takes as long whatever its rows
    if (leave_out) {
        RowsParams q{};
        q.targets = targets, q.hidden = static_cast<const __nv_bfloat16 *>(hidden), q.hidden_stride = hidden_stride, q.loss_out = loss, q.lse_out = lse, q.scale = scale;
        if (int rc = start_rows(q, plan, ws, st)) return rc;
        p.common = q.common, p.index = q.index, p.rows = q.rows;
    } else {
        p.targets = targets;
    }
    if (int rc = start_either<LossTask>(plan.pairs_logits, maps, p, tiles_of(rows, side) * tiles_of(vocab, side), st, leave_out)) return rc;
    KT_CUDA(launch_behind(k_xent_join, 1, dim3(static_cast<unsigned>((rows + 7) / 8)), dim3(256), 0, st, p, static_cast<int>(tiles_of(vocab, side / 2)), loss, lse));
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

    LogitsMaps logits{};
    BackMaps back{};
    if (int rc = describe_rows(&logits.hidden, &logits.packed, plan, hidden, hidden_stride, ws, false)) return rc;
    if (int rc = describe_operand(&logits.weight, "weight", false, false, weight, dim, vocab, 1, weight_stride * 2, 0)) return rc;
    if (int rc = describe_matrix(&logits.p, "the workspace", CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0, 64, 32)) return rc;
    if (dhidden != nullptr) {
        if (int rc = describe_operand(&back.p, "the workspace", false, false, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0, rows_of_box(rows))) return rc;
        if (!direct)
            if (int rc = describe_matrix(&back.sums, "the workspace", CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, sums, dim, rows, plan.shares, dim * 4, rows * dim * 4, 32, 32)) return rc;
    }
    if (dweight != nullptr) {
        if (int rc = describe_operand(&back.p_down, "the workspace", false, true, ws + plan.at_p, plan.piece, p_rows, 1, pitch, 0)) return rc;
        if (int rc = describe_rows(&back.hidden, &back.packed, plan, hidden, hidden_stride, ws, true)) return rc;
        if (int rc = describe_operand(&back.scaled, "the workspace", false, true, ws + plan.at_scaled, dim, up(rows, K_STEP), 1, dim * 2, 0)) return rc;
        if (int rc = describe_matrix(&back.dweight, "dweight", CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dweight, dim, vocab, 1, dweight_stride * 2, 0, 64, 32)) return rc;
    }

    RowsParams q{};
    q.targets = targets, q.hidden = static_cast<const __nv_bfloat16 *>(hidden), q.hidden_stride = hidden_stride, q.scale = scale;
    q.dloss = dloss, q.dlse = dlse, q.lse = lse, q.dhidden = static_cast<__nv_bfloat16 *>(dhidden), q.dhidden_stride = dhidden_stride;
    if (int rc = start_rows(q, plan, ws, st)) return rc;
    for (int64_t i = 0; i < plan.pieces; ++i) {
        const int64_t from = i * plan.piece, past = from + plan.piece < vocab ? from + plan.piece : vocab;
        LogitsParams p{};
        p.common = q.common, p.rows = q.rows, p.n = q.n, p.vocab = q.vocab, p.steps = static_cast<int>((dim + K_STEP - 1) / K_STEP);
        p.from = static_cast<int>(from), p.past = static_cast<int>(past), p.band = band_of(dim, plan.pairs_logits ? 256 : 128), p.scale_log2 = scale * LOG2E;
        const int64_t columns = past - from;
        const int side = plan.pairs_logits ? 256 : 128, back_side = plan.pairs_back ? 256 : 128;
        if (int rc = start_either<GradTask>(plan.pairs_logits, logits, p, tiles_of(rows, side) * tiles_of(columns, side), st)) return rc;
        if (dhidden != nullptr)       // the weights' rows from the piece's first on
            if (int rc = describe_operand(&back.weight, "weight", false, true, static_cast<const __nv_bfloat16 *>(weight) + from * weight_stride, dim, columns, 1, weight_stride * 2, 0)) return rc;
        BackParams b{};
        b.common = q.common, b.index = q.index, b.units = q.units, b.to = direct ? q.dhidden : nullptr, b.to_stride = dhidden_stride, b.n = q.n, b.dim = q.dim, b.from = p.from, b.past = p.past;
        b.tiles_n = static_cast<int>(tiles_of(dim, back_side)), b.tiles_w = dweight != nullptr ? static_cast<int>(tiles_of(columns, back_side)) : 0;
        b.shares = static_cast<int>(plan.shares), b.steps = static_cast<int>(tiles_of(columns, K_STEP)), b.add = i > 0, b.hidden = dhidden != nullptr;
        const int64_t tiles = (dhidden != nullptr ? tiles_of(rows, back_side) * b.tiles_n * plan.shares : 0) + static_cast<int64_t>(b.tiles_w) * b.tiles_n;
        if (int rc = start_either<BackTask>(plan.pairs_back, back, b, tiles, st)) return rc;
    }
    if (dhidden != nullptr && !direct) {
        const int64_t blocks = (rows * (dim / 8) + 255) / 256;
        KT_CUDA(launch_behind(k_xent_dhidden, 1, dim3(static_cast<unsigned>(blocks < 8 * PRODUCT_SMS ? blocks : 8 * PRODUCT_SMS)), dim3(256), 0, st, static_cast<const Common *>(q.common),
                              static_cast<const int *>(q.index), static_cast<const float *>(q.units), static_cast<const float *>(sums), static_cast<int>(plan.shares), rows * dim, q.dim, q.dhidden, dhidden_stride));
    }
    return KT_OK;
}

}  // extern "C"
