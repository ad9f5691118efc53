// kt_attn.cu -- softmax attention and its backward pass on bf16 heads, for the training step whose
// gradients the library synchronises.  Contracts: include/kaitian.h.
//
// With S = scale Q K^T under the mask, lse_i = log sum_j exp(S_ij) and P = exp(S - lse):
//   forward    O = P V, one pass over the keys with a running maximum and sum per query
//   backward   delta_i = sum_d dO_id O_id,  dP = dO V^T,  dS = P (dP - delta),
//              dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
// The backward pass recomputes P from Q, K and lse, twice: one CTA per 128 queries goes over the keys (dQ), one
// per 128 keys over the queries of all heads that share them (dK, dV).  Every sum has one owner, so nothing
// is added with atomics and the result does not depend on the order in which CTAs run; the price is that
// S and dP are formed twice (7 products, not 5).
//
// All products run on the tensor cores (kt_tensor.cuh): operands come in by tile copies, sums stay in
// tensor memory, and the probabilities (dS) go back to tensor memory as bf16, where they are the first
// operand of the next product.  One warp brings tiles, three issue products, eight compute.
// Rows past a sequence's length may hold anything: they are cleared in shared memory where they would
// be multiplied by a zero.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstddef>

#include "kt_internal.h"
#include "kt_pairs.cuh"
#include "kt_tensor.cuh"

using namespace ktd;

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// The third group of warps: one brings tiles, the others issue products, each its own kind.  What a thread issues
// after a product waits until that has all but run (measured: some 500 cycles for 8 instructions of 64), so
// a thread that then waited for a barrier would leave the tensor cores idle meanwhile; another has queued its
// product by then.
constexpr int WARP_SCORES = 8, WARP_LOAD = 9, WARP_DP = 10, WARP_SUMS = 11, THREADS = 384;
// Registers: a block of 384 threads starts with 168 each, 64512 in all; the third group gives back what the
// eight warps that compute take: 256 x 208 + 128 x 88 = 64512.
constexpr int REGISTERS_COMPUTE = 208, REGISTERS_HELP = 88;
constexpr uint32_t TMEM_COLUMNS = 512;
constexpr int SMS = 148;                        // of a B200, one CTA to each

struct QueryStats;

struct AttnParams {
    const int32_t *used_q, *used_kv;
    const __nv_bfloat16 *o, *dout;
    __nv_bfloat16 *out, *dk, *dv;               // O or dQ
    float *lse;
    QueryStats *stats;
    unsigned *next_item;
    int64_t o_stride[3], dout_stride[3], out_stride[3], dk_stride[3], dv_stride[3];     // batch, token, head
    int batch, heads, heads_kv, len_q, len_kv, dim, causal;
    int tiles_q, tiles_kv, parts;               // parts: CTAs that share a work item, where they do
    float scale, scale_log2;
    uint64_t wait_ns;                           // how long a wait may last
};

// Tokens in use of a sequence, and how far a query sees.
struct Seq {
    int n, m, shift, causal;                    // queries, keys, m - n
    __device__ Seq(const AttnParams &p, int b) {
        n = p.used_q ? min(max(p.used_q[b], 0), p.len_q) : p.len_q;
        m = p.used_kv ? min(max(p.used_kv[b], 0), p.len_kv) : p.len_kv;
        shift = m - n;
        causal = p.causal;
    }
    __device__ int keys_of(int i) const { return i >= n ? 0 : causal ? max(0, min(m, i + 1 + shift)) : m; }      // keys 0 ... of query i
    __device__ int first_query_of(int j) const { return causal ? max(0, j - shift) : 0; }                    // the first that sees key j
};

__device__ __forceinline__ int tiles(int rows) { return (rows + TILE - 1) / TILE; }

// One tile [128 tokens x DH] into shared memory; `full` is arrived at once it is there.  Rows from `used`
// on that lie inside the tensor (`len`) hold whatever the caller left there: with CLEAN they are
// cleared first, which the whole warp does (rows past `len` arrive as zeros).
template <int DH, bool CLEAN>
__device__ __forceinline__ bool load_tile(uint32_t to, uint8_t *to_ptr, const CUtensorMap *map, uint64_t *full, uint64_t *landed, uint32_t &landed_phase,
                                          int token, int used, int len, int head, int batch, volatile Patience *waits) {
    const int lane = threadIdx.x % 32;
    const bool dirty = CLEAN && used < min(len, token + TILE);
    uint64_t *bar = dirty ? landed : full;
    if (lane == 0) {
        bar_expect(bar, DH / 64 * CHUNK);
#pragma unroll
        for (int c = 0; c < DH / 64; ++c) copy_tile(to + c * CHUNK, map, bar, c * 64, token, head, batch);
    }
    __syncwarp();
    if (!dirty) return true;
    if (!bar_wait(landed, landed_phase, waits)) return false;
    landed_phase ^= 1;
    const int from = max(0, used - token);
    for (int i = from * 8 + lane; i < TILE * 8; i += 32)
#pragma unroll
        for (int c = 0; c < DH / 64; ++c) *reinterpret_cast<uint4 *>(to_ptr + c * CHUNK + i * 16) = make_uint4(0, 0, 0, 0);
    fence_async_smem();
    __syncwarp();
    if (lane == 0) bar_arrive(full);
    return true;
}

// 32 columns of a row, scaled, as bf16 to `row` (columns from c0 on that exist).
__device__ __forceinline__ void write_columns(__nv_bfloat16 *row, int c0, int dim, const uint32_t (&r)[32], float by) {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
        if (c0 + c < dim) {
            uint4 v;
            v.x = pack_bf16(__uint_as_float(r[c]) * by, __uint_as_float(r[c + 1]) * by);
            v.y = pack_bf16(__uint_as_float(r[c + 2]) * by, __uint_as_float(r[c + 3]) * by);
            v.z = pack_bf16(__uint_as_float(r[c + 4]) * by, __uint_as_float(r[c + 5]) * by);
            v.w = pack_bf16(__uint_as_float(r[c + 6]) * by, __uint_as_float(r[c + 7]) * by);
            *reinterpret_cast<uint4 *>(row + c0 + c) = v;
        }
    }
}
__device__ __forceinline__ void write_zeros(__nv_bfloat16 *row, int c0, int c1) {
    for (int c = c0; c < c1; c += 8) *reinterpret_cast<uint4 *>(row + c) = make_uint4(0, 0, 0, 0);
}

// The end of a CTA one of whose waits has given up.  Copies, products and answers in flight get two milliseconds to
// finish before the memory that they write is handed back.  Then all results of the call become NaN (fill_nan, by the
// eight warps that compute): the CTA has taken items that nobody else will do, and what others write later is right.
__device__ __forceinline__ void settle() {
    const uint64_t start = now_ns();
    for (int i = 0; i < 100000 && now_ns() - start < 2000000; ++i) __nanosleep(1000);
}
__device__ __forceinline__ void fill_nan(__nv_bfloat16 *at, const int64_t (&stride)[3], int batch, int tokens, int heads, int dim) {
    const int64_t pieces = dim / 8, all = static_cast<int64_t>(batch) * tokens * heads * pieces;
    for (int64_t i = threadIdx.x; i < all; i += 256) {
        const int64_t row = i / pieces, token = row / heads;
        *reinterpret_cast<uint4 *>(at + token / tokens * stride[0] + token % tokens * stride[1] + row % heads * stride[2] + i % pieces * 8) =
            make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);
    }
}

// ------------------------------------------------------------------------------------ forward
// Two tiles of 128 queries to a work item, four warps on each.  A thread owns a row: maximum and sum need
// no exchange.  A group takes its scores into registers at once, and their place in tensor memory is free for
// the other group's next ones, so that neither a group nor the tensor cores wait for the other in turn.
// CTAs stay (Queue): the next item's tiles are fetched and its first scores formed while the last item's
// output is written, which short sequences need most.  Every barrier's phases are counted on from item to item.
// With SPLIT, for few long items, the CTAs of a cluster share the keys of one item and join what each has of it
// through distributed shared memory: no workspace, and the same bits every time.
// Tensor memory: scores 0, probabilities 128 and 192, sums 256 and 256 + DH.
// 8192 tokens causal, 16 heads of 128 on 4: 208 us, 1320 TFLOP/s, where a large library product reaches 1650 in a burst and
// 1406 at the power limit, which this meets as well.  Short sequences and heads of 64 wait for exponentials (a step of 128
// keys takes some 1.5 us whatever the head's size): 4 x 333, 12 heads of 80 on 4 in 12 us.
template <int DH>
struct FwdSmem {
    static constexpr uint32_t TILE_BYTES = DH / 64 * CHUNK;
    static constexpr int SETS = DH == 64 ? 2 : 1, K_SLOTS = 3, V_SLOTS = 2;       // of query tiles: two where there is room
    alignas(1024) uint8_t q[SETS][2][TILE_BYTES], k[K_SLOTS][TILE_BYTES], v[V_SLOTS][TILE_BYTES];
    Queue queue;
    uint64_t q_full[SETS], q_free[SETS], k_full[K_SLOTS], k_free[K_SLOTS], v_full[V_SLOTS], v_free[V_SLOTS], s_full[2], s_taken, p_ready[2], o_done[2], o_taken[2], landed;
    uint32_t tmem;
    Patience waits;
};

// What a CTA takes of n steps that the CTAs of its cluster share.
__device__ __forceinline__ void take_share(const AttnParams &p, int &from, int &n) {
    const int64_t rank = blockIdx.x % p.parts, all = n;
    from = static_cast<int>(all * rank / p.parts);
    n = static_cast<int>(all * (rank + 1) / p.parts) - from;
}

// Sums of a row in fp32, 32 columns at a time, to where the others of the cluster read them.  Rows follow
// one another; the 16-byte pieces of 32 columns change places from row to row, so that neighbours meet different banks.
__device__ __forceinline__ void put_sums(void *tiles, int dh, int row, int c, const uint32_t (&o)[32], bool zeros) {
    float4 *const to = static_cast<float4 *>(tiles) + row * (dh / 4) + c / 4;
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (!zeros) v = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]));
        to[e / 4 ^ row % 8] = v;
    }
}
// 8 columns of it, v = 0 or 1: the first four or the others.
__device__ __forceinline__ float4 get_sums(uint32_t tiles, int dh, int row, int c8, int v, unsigned rank) {
    return of_cta4(tiles + row * dh * 4 + (2 * c8 / 8 * 8 + ((2 * c8 + v) % 8 ^ row % 8)) * 16, rank);
}

// A work item: the pair of query tiles, and the key tiles that each of them sees; with SPLIT, a CTA's share of these.
template <bool SPLIT>
struct FwdItem {
    int row0, b, h, h_kv, from, n_tiles[2], n, common, longer, steps;
    __device__ FwdItem(const AttnParams &p, int block) {
        const int pairs = (p.tiles_q + 1) / 2, all = p.batch * p.heads, bh = block % all;
        row0 = (pairs - 1 - block / all) * 2 * TILE;               // the longest rows first
        b = bh / p.heads, h = bh % p.heads, h_kv = h / (p.heads / p.heads_kv);
        const Seq seq(p, b);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int first = row0 + w * TILE;
            n_tiles[w] = first < seq.n ? tiles(seq.keys_of(min(first + TILE, seq.n) - 1)) : 0;
        }
        n = max(n_tiles[0], n_tiles[1]), from = 0;
        if constexpr (SPLIT) {
            take_share(p, from, n);
#pragma unroll
            for (int w = 0; w < 2; ++w) n_tiles[w] = max(0, min(n_tiles[w] - from, n));
        }
        // Steps: the two tiles in turn while both have keys left, then the one that has more.
        common = min(n_tiles[0], n_tiles[1]), longer = n_tiles[1] > n_tiles[0] ? 1 : 0, steps = n_tiles[0] + n_tiles[1];
    }
    __device__ int key_tile(int u) const { return u < 2 * common ? u / 2 : u - common; }
    __device__ int group(int u) const { return u < 2 * common ? u & 1 : longer; }
    __device__ bool last_use(int u) const { return group(u) == 1 || key_tile(u) >= n_tiles[1]; }      // of its key tile
};

// A row of a split item: sums O_r and s_r over share r of the keys, taken with maxima m_r, give
// O = (sum_r 2^(m_r - m) O_r) / (sum_r 2^(m_r - m) s_r) with m the largest.  Every CTA of the cluster takes its share of the
// rows, reads them from all, in their order, and writes them; 8 columns to a thread.
template <int DH, int PARTS>
__device__ __forceinline__ void join_parts(const AttnParams &p, const FwdItem<true> &it, uint32_t at) {
    static_assert(2 * TILE * (DH * 4 + 8) <= offsetof(FwdSmem<DH>, queue));
    constexpr int LANES = DH / 8, SHARE = 2 * TILE / PARTS;
    const int from = blockIdx.x % PARTS * SHARE, c = threadIdx.x % LANES;
    for (int r = from + threadIdx.x / LANES; r < from + SHARE; r += 2 * TILE / LANES) {
        const int row = it.row0 + r;
        if (row >= p.len_q) break;
        const uint32_t stats = at + 2 * TILE * DH * 4 + r * 8;
        float2 s[PARTS];
        float4 x[PARTS][2];                     // all on their way before the first is used
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            s[i] = of_cta2(stats, i);
#pragma unroll
            for (int e = 0; e < 2; ++e) x[i][e] = get_sums(at, DH, r, c, e, i);
        }
        float top = -INFINITY, sum = 0.0f, o[8] = {};
#pragma unroll
        for (int i = 0; i < PARTS; ++i) top = fmaxf(top, s[i].x);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            const float by = s[i].y == 0.0f ? 0.0f : exp2_fast(s[i].x - top);
            sum = fmaf(s[i].y, by, sum);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                o[e * 4] = fmaf(x[i][e].x, by, o[e * 4]), o[e * 4 + 1] = fmaf(x[i][e].y, by, o[e * 4 + 1]);
                o[e * 4 + 2] = fmaf(x[i][e].z, by, o[e * 4 + 2]), o[e * 4 + 3] = fmaf(x[i][e].w, by, o[e * 4 + 3]);
            }
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (c * 8 < p.dim)
            *reinterpret_cast<uint4 *>(p.out + it.b * p.out_stride[0] + row * p.out_stride[1] + it.h * p.out_stride[2] + c * 8) =
                make_uint4(pack_bf16(o[0] * by, o[1] * by), pack_bf16(o[2] * by, o[3] * by), pack_bf16(o[4] * by, o[5] * by), pack_bf16(o[6] * by, o[7] * by));
        if (c == 0) p.lse[(static_cast<int64_t>(it.b) * p.heads + it.h) * p.len_q + row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
}

template <int DH, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
k_attn_forward(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
               const AttnParams p) {
    extern __shared__ uint8_t raw[];
    using Smem = FwdSmem<DH>;
    using Item = FwdItem<SPLIT>;
    constexpr int SETS = Smem::SETS, K_SLOTS = Smem::K_SLOTS, V_SLOTS = Smem::V_SLOTS;
    auto &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        queue_init(sm.queue, 3 + 8);
        for (int i = 0; i < SETS; ++i) bar_init(&sm.q_full[i], 1), bar_init(&sm.q_free[i], 1);
        for (int i = 0; i < K_SLOTS; ++i) bar_init(&sm.k_full[i], 1), bar_init(&sm.k_free[i], 1);
        for (int i = 0; i < V_SLOTS; ++i) bar_init(&sm.v_full[i], 1), bar_init(&sm.v_free[i], 1);
        for (int w = 0; w < 2; ++w) bar_init(&sm.s_full[w], 1), bar_init(&sm.p_ready[w], 4), bar_init(&sm.o_done[w], 1), bar_init(&sm.o_taken[w], 4);
        bar_init(&sm.s_taken, 4), bar_init(&sm.landed, 1);
        sm.waits = {p.wait_ns, 0};
        fence_async_smem();
    }
    if (warp == WARP_SCORES) tmem_alloc(&sm.tmem, TMEM_COLUMNS);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = sm.tmem;
    const int first_block = SPLIT ? blockIdx.x / p.parts : blockIdx.x;       // and the only one, with SPLIT
    volatile Patience *waits = &sm.waits;

    if (warp == WARP_LOAD) {
        registers_give<REGISTERS_HELP>();
        uint32_t asked = 0, sets = 0, tiles_in = 0, landed_phase = 0;      // counts over all items
        bool ok = true;
        for (int block = first_block; ok && block >= 0; block = SPLIT ? -1 : queue_next<false>(sm.queue, asked - 1, waits)) {
            const Item it(p, block);
            const Seq seq(p, it.b);
            if constexpr (!SPLIT) {
                if (!(ok = bar_wait(&sm.queue.free[asked % QUEUE], (asked / QUEUE + 1) & 1, waits))) break;
                if (lane == 0) queue_ask(sm.queue, asked);
                ++asked;
            }
            if (it.n == 0) continue;
            const int set = sets % SETS;
            if (!(ok = bar_wait(&sm.q_free[set], (sets / SETS + 1) & 1, waits))) break;
            ++sets;
            if (lane == 0) {
                bar_expect(&sm.q_full[set], 2 * Smem::TILE_BYTES);
                for (int w = 0; w < 2; ++w)
                    for (int c = 0; c < DH / 64; ++c) copy_tile(smem_addr(sm.q[set][w]) + c * CHUNK, &map_q, &sm.q_full[set], c * 64, it.row0 + w * TILE, it.h, it.b);
            }
            __syncwarp();
            for (int j = 0; ok && j <= it.n; ++j) {              // keys a tile ahead of values
                if (j < it.n) {
                    const uint32_t i = tiles_in + j, ks = i % K_SLOTS;
                    ok = bar_wait(&sm.k_free[ks], (i / K_SLOTS + 1) & 1, waits) &&
                         load_tile<DH, false>(smem_addr(sm.k[ks]), sm.k[ks], &map_k, &sm.k_full[ks], &sm.landed, landed_phase, (it.from + j) * TILE, seq.m, p.len_kv, it.h_kv, it.b, waits);
                }
                if (ok && j > 0) {
                    const uint32_t i = tiles_in + j - 1, vs = i % V_SLOTS;
                    ok = bar_wait(&sm.v_free[vs], (i / V_SLOTS + 1) & 1, waits) &&
                         load_tile<DH, true>(smem_addr(sm.v[vs]), sm.v[vs], &map_v, &sm.v_full[vs], &sm.landed, landed_phase, (it.from + j - 1) * TILE, seq.m, p.len_kv, it.h_kv, it.b, waits);
                }
            }
            tiles_in += it.n;
        }
    } else if (warp == WARP_SCORES) {
        registers_give<REGISTERS_HELP>();
        if (elected()) {
            const uint32_t q_at = smem_addr(sm.q), k_at = smem_addr(sm.k);
            uint32_t items = 0, sets = 0, tiles_in = 0, steps = 0;
            bool ok = true;
            for (int block = first_block; ok && block >= 0; block = SPLIT ? -1 : queue_next_one<false>(sm.queue, items++, waits)) {
                const Item it(p, block);
                if (it.n == 0) continue;
                const uint32_t set = sets % SETS;
                ok = bar_wait_one(&sm.q_full[set], sets / SETS & 1, waits);
                ++sets;
                for (int u = 0; ok && u < it.steps; ++u, ++steps) {
                    const int w = it.group(u);
                    const uint32_t i = tiles_in + it.key_tile(u), ks = i % K_SLOTS;
                    ok = bar_wait_one(&sm.k_full[ks], i / K_SLOTS & 1, waits) && (steps == 0 || bar_wait_one(&sm.s_taken, (steps - 1) & 1, waits));
                    if (!ok) break;
                    tmem_fence_after();
                    product_rows<DH, TILE>(tmem, q_at + (set * 2 + w) * Smem::TILE_BYTES, k_at + ks * Smem::TILE_BYTES);
                    mma_commit(&sm.s_full[w]);
                    if (it.last_use(u)) mma_commit(&sm.k_free[ks]);
                    if (u == it.steps - 1) mma_commit(&sm.q_free[set]);
                }
                tiles_in += it.n;
            }
        }
        __syncwarp();
    } else if (warp == WARP_SUMS) {
        registers_give<REGISTERS_HELP>();
        if (elected()) {
            const uint32_t v_at = smem_addr(sm.v);
            uint32_t items = 0, tiles_in = 0, mine[2] = {0, 0}, outputs[2] = {0, 0};
            bool ok = true;
            for (int block = first_block; ok && block >= 0; block = SPLIT ? -1 : queue_next_one<false>(sm.queue, items++, waits)) {
                const Item it(p, block);
                for (int u = 0; ok && u < it.steps; ++u) {
                    const int w = it.group(u), j = it.key_tile(u);
                    const uint32_t i = tiles_in + j, vs = i % V_SLOTS;
                    ok = bar_wait_one(&sm.v_full[vs], i / V_SLOTS & 1, waits) && bar_wait_one(&sm.p_ready[w], (mine[w] + j) & 1, waits) &&
                         (j > 0 || outputs[w] == 0 || bar_wait_one(&sm.o_taken[w], (outputs[w] - 1) & 1, waits));       // the last item's sums have been read
                    if (!ok) break;
                    tmem_fence_after();
                    product_down<DH, TILE>(tmem + 256 + w * DH, tmem + TILE + w * 64, v_at + vs * Smem::TILE_BYTES, j > 0);
                    mma_commit(&sm.o_done[w]);
                    if (it.last_use(u)) mma_commit(&sm.v_free[vs]);
                }
                tiles_in += it.n;
                for (int w = 0; w < 2; ++w) mine[w] += it.n_tiles[w], outputs[w] += it.n_tiles[w] > 0;
            }
        }
        __syncwarp();
    } else if (warp < 8) {
        registers_take<REGISTERS_COMPUTE>();
        const int w = warp / 4;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16), s_at = lanes, p_at = lanes + TILE + w * 64, o_at = lanes + 256 + w * DH;
        uint32_t items = 0, mine = 0;
        bool ok = true;
        for (int block = first_block; ok && block >= 0; block = SPLIT ? -1 : queue_next<false>(sm.queue, items++, waits)) {
            const Item it(p, block);
            const Seq seq(p, it.b);
            const int row = it.row0 + w * TILE + threadIdx.x % TILE, n_mine = w == 0 ? it.n_tiles[0] : it.n_tiles[1];
            const int limit = seq.keys_of(row), all_see = seq.keys_of(it.row0 + w * TILE);    // the tile's first row sees least
            const bool whole = it.row0 + w * TILE + TILE <= seq.n;
            float top = -INFINITY, sum = 0.0f;      // in units of log 2, after scaling
            for (int j = 0; j < n_mine; ++j) {
                const uint32_t i = mine + j;
                if (!(ok = bar_wait(&sm.s_full[w], i & 1, waits))) break;
                tmem_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int q = 0; q < 4; ++q) tmem_load32(s_at + q * 32, s[q]);
                tmem_wait_loads(s);
                tmem_fence_before();
                bar_arrive_warp(&sm.s_taken);
                if (!whole || (it.from + j + 1) * TILE > all_see) {
                    const int left = limit - (it.from + j) * TILE;           // columns that the row sees
#pragma unroll
                    for (int c = 0; c < TILE; ++c)
                        if (c >= left) s[c / 32][c % 32] = __float_as_uint(-INFINITY);
                }
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < TILE; ++c) m[c % 4] = fmaxf(m[c % 4], __uint_as_float(s[c / 32][c % 32]));
                const float here = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * p.scale_log2;
                // The running maximum follows only when it would grow by 2^8: until then probabilities of up
                // to 256 are as exact, and the sums in tensor memory need not be rescaled.
                const bool grow = here > top + 8.0f || (top == -INFINITY && here > -INFINITY);
                if (__any_sync(0xFFFFFFFFu, grow)) {
                    const float by = grow ? exp2_fast(top - here) : 1.0f;
                    if (grow) top = here;
                    sum *= by;
                    if (j > 0) {
                        if (!(ok = bar_wait(&sm.o_done[w], (i - 1) & 1, waits))) break;
                        tmem_fence_after();
#pragma unroll
                        for (int c = 0; c < DH; c += 32) {
                            uint32_t o[32];
                            tmem_load32(o_at + c, o);
                            tmem_wait_loads(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                            tmem_store32(o_at + c, o);
                        }
                    }
                }
                const float ref = top == -INFINITY ? 0.0f : top;
                float2 part[2] = {both(0.0f), both(0.0f)};
                uint32_t packed[2][32];
#pragma unroll
                for (int c = 0; c < TILE; c += 2) {
                    const float2 x = fma2(pair_of(s[c / 32], c % 32), both(p.scale_log2), both(-ref));
                    const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
                    part[c / 2 % 2] = add2(part[c / 2 % 2], e);
                    packed[c / 64][c % 64 / 2] = pack_bf16(e);
                }
                if (j > 0) {                        // the last probabilities have been used
                    if (!(ok = bar_wait(&sm.o_done[w], (i - 1) & 1, waits))) break;
                    tmem_fence_after();
                }
                tmem_store32(p_at, packed[0]);
                tmem_store32(p_at + 32, packed[1]);
                sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                tmem_wait_stores();
                tmem_fence_before();
                bar_arrive_warp(&sm.p_ready[w]);
            }
            mine += n_mine;
            if constexpr (SPLIT) {                  // what the CTA has of the row, over the tiles that are done with
                if (ok && n_mine > 0) ok = bar_wait(&sm.o_done[w], (mine - 1) & 1, waits);
                tmem_fence_after();
                asm volatile("barrier.sync 1, 256;" ::: "memory");
#pragma unroll
                for (int c = 0; c < DH; c += 32) {
                    uint32_t o[32];
                    tmem_load32(o_at + c, o);        // (whatever is there if the CTA has no keys)
                    tmem_wait_loads(o);
                    put_sums(&sm, DH, threadIdx.x, c, o, sum == 0.0f);
                }
                reinterpret_cast<float2 *>(reinterpret_cast<float *>(&sm) + 2 * TILE * DH)[threadIdx.x] = make_float2(top, sum);
                break;
            }
            __nv_bfloat16 *out = p.out + it.b * p.out_stride[0] + row * p.out_stride[1] + it.h * p.out_stride[2];
            if (ok && n_mine > 0) {
                if (!(ok = bar_wait(&sm.o_done[w], (mine - 1) & 1, waits))) break;
                tmem_fence_after();
                const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
                for (int c = 0; c < DH; c += 64) {
                    uint32_t o[2][32];
                    tmem_load32(o_at + c, o[0]);
                    tmem_load32(o_at + c + 32, o[1]);
                    tmem_wait_loads(o);
                    if (c == DH - 64) {
                        tmem_fence_before();
                        bar_arrive_warp(&sm.o_taken[w]);
                    }
                    if (sum == 0.0f)
#pragma unroll
                        for (int e = 0; e < 64; ++e) o[e / 32][e % 32] = 0;
                    if (row < p.len_q) write_columns(out, c, p.dim, o[0], by), write_columns(out, c + 32, p.dim, o[1], by);
                }
            } else if (ok && row < p.len_q) {
                write_zeros(out, 0, p.dim);
            }
            if (ok && row < p.len_q) p.lse[(static_cast<int64_t>(it.b) * p.heads + it.h) * p.len_q + row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
        }
    } else {
        registers_give<REGISTERS_HELP>();       // WARP_DP has nothing to do here, but its group gives back together
    }
    tmem_fence_before();
    if constexpr (SPLIT) {
        cluster_sync();
        if (warp < 8) {
            const Item it(p, first_block);
            if (p.parts == 2) join_parts<DH, 2>(p, it, smem_addr(&sm));
            else if (p.parts == 4) join_parts<DH, 4>(p, it, smem_addr(&sm));
            else join_parts<DH, 8>(p, it, smem_addr(&sm));
        }
        cluster_sync();                         // the others have read what is here
    }
    __syncthreads();
    if (waits->gave_up) {
        settle();
        if (warp < 8) {
            fill_nan(p.out, p.out_stride, p.batch, p.len_q, p.heads, p.dim);
            const int64_t rows = static_cast<int64_t>(p.batch) * p.heads * p.len_q;
            for (int64_t i = threadIdx.x; i < rows; i += 256) p.lse[i] = __int_as_float(0x7FFFFFFF);
        }
    }
    if (warp == WARP_SCORES) tmem_free(tmem, TMEM_COLUMNS);
}

// ----------------------------------------------------------------------------------- backward
// What the backward kernels need of a query besides its rows, tile by tile:
//   for dQ, fp32: lse in units of log 2 (+inf where a query sees nothing or is not in use, which makes its
//   probabilities exp2(s - inf) = 0), and delta;
//   for dK and dV: -lse / scale and -delta, each as a sum of three bf16 (24 bits), side by side in 16 bytes.  There
//   queries are columns, and a thread would have to read every column's values from shared memory for
//   each row; instead the tensor cores add them: one more product over 16 elements, with a row of ones.
struct QueryStats {
    float lse[TILE], delta[TILE];
    uint4 terms[TILE];
};
constexpr float HIDDEN = -1e30f;                // in place of -lse / scale where nothing is seen

__device__ __forceinline__ void three_terms(float x, uint16_t (&to)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const __nv_bfloat16 t = __float2bfloat16_rn(x);
        to[i] = __bfloat16_as_ushort(t);
        x -= __bfloat162float(t);
    }
}

// A tile to a CTA, LANES neighbours to a row.  Bound by memory: O and dO are read once, all of a thread's
// vectors before the first is used (16 heads of 8192 x 128: 15 us, 4400 GB/s).
template <int LANES>
__global__ void __launch_bounds__(256) k_attn_stats(const AttnParams p) {
    constexpr int ROWS = 256 / LANES, PASSES = TILE / ROWS;
    const int bh = blockIdx.x / p.tiles_q, tile = blockIdx.x % p.tiles_q, b = bh / p.heads, h = bh % p.heads;
    const int lane = threadIdx.x % LANES, in_pass = threadIdx.x / LANES;
    let_next_begin();
    const Seq seq(p, b);
    const __nv_bfloat16 *o = p.o + b * p.o_stride[0] + h * p.o_stride[2] + lane * 8, *dout = p.dout + b * p.dout_stride[0] + h * p.dout_stride[2] + lane * 8;
    __shared__ float deltas[TILE];
    float lse = -INFINITY;
    if (threadIdx.x < TILE && tile * TILE + static_cast<int>(threadIdx.x) < seq.n) lse = p.lse[static_cast<int64_t>(bh) * p.len_q + tile * TILE + threadIdx.x];
    uint4 x[PASSES], y[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int64_t row = tile * TILE + i * ROWS + in_pass;
        x[i] = y[i] = make_uint4(0, 0, 0, 0);
        if (row < seq.n && lane * 8 < p.dim) {
            x[i] = *reinterpret_cast<const uint4 *>(o + row * p.o_stride[1]);
            y[i] = *reinterpret_cast<const uint4 *>(dout + row * p.dout_stride[1]);
        }
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, v[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
        float delta = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            delta = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(v[e] << 16), delta);
            delta = fmaf(__uint_as_float(u[e] & 0xFFFF0000u), __uint_as_float(v[e] & 0xFFFF0000u), delta);
        }
#pragma unroll
        for (int d = LANES / 2; d > 0; d /= 2) delta += __shfl_xor_sync(0xFFFFFFFFu, delta, d);
        if (lane == 0) deltas[i * ROWS + in_pass] = delta;
    }
    __syncthreads();
    if (threadIdx.x < TILE) {
        const bool empty = lse == -INFINITY;
        const float delta = empty ? 0.0f : deltas[threadIdx.x];
        QueryStats &to = p.stats[blockIdx.x];
        to.lse[threadIdx.x] = empty ? INFINITY : lse * LOG2E;
        to.delta[threadIdx.x] = delta;
        uint16_t l[3], d[3];
        three_terms(empty ? HIDDEN : -lse / p.scale, l);
        three_terms(-delta, d);
        to.terms[threadIdx.x] = make_uint4(l[0] | l[1] << 16, l[2] | d[0] << 16, d[1] | d[2] << 16, 0);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.next_item = 0;
}

// The backward pass in one launch, whose CTAs stay (Queue, with a counter: a CTA must not be handed a key tile
// after a query tile): first the key tiles, whose work is the larger, then
// the query tiles, each kind in the order of what a causal mask leaves it.  A CTA does key tiles until
// it is handed its first query tile.  Barriers of both kinds are made at the start, and their phases are
// counted on from item to item: the next item's tiles are fetched and its first products formed
// while the last one's sums are written.
// 8192 tokens causal, 16 heads of 128 on 4: 718 us, 955 TFLOP/s by the formulas' five products, 1335 by the seven that are
// formed, at the power limit.  8 x 1024 causal, 16 heads of 64: 134 us; there a product of 64 columns costs as much as one
// of 128, and the two groups' exponentials and the ends of items take the rest.
struct DqBars {
    static constexpr int K_MOST = 5, V_MOST = 3;
    uint64_t q_full[2], q_free[2], k_full[K_MOST], k_free[K_MOST], v_full[V_MOST], v_free[V_MOST], s_full[2], s_taken, dp_full[2], dp_taken, ds_ready[2], dq_done[2], sums_full, sums_taken;
};
struct DkvBars {
    static constexpr int Q_MOST = 4, DO_MOST = 3;
    uint64_t kv_full[2], kv_free[2], q_full[Q_MOST], q_free[Q_MOST], do_full[DO_MOST], do_free[DO_MOST], s_full[2], s_taken, dp_full[2], dp_taken, p_ready[2], ds_ready[2], dv_done[2], dk_done[2],
        sums_full, sums_taken;
};
struct BwdCommon {
    Queue queue;
    DqBars dq;
    DkvBars dkv;
    uint64_t landed;
    uint32_t tmem;
    Patience waits;
};
constexpr uint32_t QUEUE_READERS = 4 + 8;       // the four warps of the third group, the eight that compute

// dQ: 128 queries to an item, the two groups of four warps take its key tiles in turn (counted over all
// items).  Scores and dP are taken into registers as soon as they are there, which frees their place for the
// next tile's.  Tensor memory: scores 0, dP 128, dS 256 and 320, sums 384.
template <int DH>
struct DqTiles {
    static constexpr uint32_t TILE_BYTES = DH / 64 * CHUNK;
    static constexpr int SETS = DH == 64 ? 2 : 1, K_SLOTS = DH == 64 ? 5 : 3, V_SLOTS = DH == 64 ? 3 : 2;
    alignas(1024) uint8_t q[SETS][TILE_BYTES], dout[SETS][TILE_BYTES], k[K_SLOTS][TILE_BYTES], v[V_SLOTS][TILE_BYTES];
};

struct DqItem {
    int tile, row0, b, h, h_kv, bh, n;          // n: key tiles
    __device__ DqItem(const AttnParams &p, int block) {
        const int all = p.batch * p.heads;
        bh = block % all, tile = p.tiles_q - 1 - block / all, row0 = tile * TILE;
        b = bh / p.heads, h = bh % p.heads, h_kv = h / (p.heads / p.heads_kv);
        const Seq seq(p, b);
        n = row0 < seq.n ? tiles(seq.keys_of(min(row0 + TILE, seq.n) - 1)) : 0;
    }
};

// dK and dV: 128 keys to an item, which goes over the query tiles of every head that shares them.  All products
// are taken transposed (rows are keys), so that P^T and dS^T are first operands from tensor memory.  Scores
// and dP are taken into registers as soon as they are there.
//   Heads of up to 64: the groups of four warps take tiles in turn.  Tensor memory: scores 0, dP 128, a
//   place of each group for P and then, once that is used, dS 256 and 320, sums 384 and 448.
//   Heads of up to 128, whose sums fill half of tensor memory: both groups work on one tile, 64 queries each.
//   A tile has a place, 0 or 128 in turn, that its scores, then dP, then P and dS take; sums 256 and 384.  Exponentials are
//   taken while the products with the last tile's P and dS run; only dP is waited for.  (The next tile but one gets
//   the place when these products have ended, which nothing else would order.  With one place for the dP of all
//   tiles every tile waited for that end: 2048 tokens causal, 8 heads of 128 on 1, in 72 us, now 67.)
// (Steps of 64 queries would leave room for turns there too, but a product of fewer than 128 columns takes
// as long as one of 128.)
template <int DH>
struct DkvTiles {
    static constexpr uint32_t TILE_BYTES = DH / 64 * CHUNK;
    static constexpr bool TURNS = DH == 64;
    static constexpr uint32_t MINE = 2 * TILE, DV = TURNS ? 384 : 256, DK = DV + DH;
    __device__ static uint32_t scores(uint32_t g) { return TURNS ? 0 : (g & 1) * TILE; }            // of the g-th query tile
    __device__ static uint32_t dprobs(uint32_t g) { return TURNS ? TILE : (g & 1) * TILE; }
    static constexpr int SETS = TURNS ? 2 : 1, Q_SLOTS = TURNS ? 4 : 2, DO_SLOTS = TURNS ? 3 : 2;
    alignas(1024) uint8_t k[SETS][TILE_BYTES], v[SETS][TILE_BYTES], q[Q_SLOTS][TILE_BYTES], dout[DO_SLOTS][TILE_BYTES];
    alignas(128) uint4 ones_lse[TILE], ones_delta[TILE], terms[Q_SLOTS][TILE], zeros[TILE];      // zeros come last: product_short
};

template <bool SPLIT>
struct DkvItem {
    int key0, b, h_kv, shared, first, per_head, from, n;       // query tiles: from `first` on, so many to a head; of those of all heads, n from `from` on
    __device__ DkvItem(const AttnParams &p, int block) {
        const int all = p.batch * p.heads_kv, bh = block % all;
        key0 = block / all * TILE;                        // early keys are seen most
        b = bh / p.heads_kv, h_kv = bh % p.heads_kv, shared = p.heads / p.heads_kv;
        const Seq seq(p, b);
        first = seq.first_query_of(key0) / TILE;
        per_head = key0 < seq.m ? max(0, tiles(seq.n) - first) : 0;
        n = per_head * shared, from = 0;
        if constexpr (SPLIT) take_share(p, from, n);
    }
};

template <int DH>
struct BwdSmem {
    union {
        DqTiles<DH> dq;
        DkvTiles<DH> dkv;
    };
    BwdCommon common;
};

// With SPLIT, where key tiles are few, the CTAs of a cluster share the queries of one and add their sums, each those of its
// share of the rows (dV and dK of 128 keys), always in the same order; then they go on with the query tiles.
template <int DH, int PARTS>
__device__ __forceinline__ void join_sums(const AttnParams &p, int block, uint32_t at) {
    static_assert(2 * TILE * DH * 4 <= offsetof(BwdSmem<DH>, common));
    constexpr int LANES = DH / 8, SHARE = 2 * TILE / PARTS;
    const int from = blockIdx.x % PARTS * SHARE, c = threadIdx.x % LANES;
    const DkvItem<true> it(p, block);
    for (int r = from + threadIdx.x / LANES; r < from + SHARE; r += 2 * TILE / LANES) {
        const bool dv = r < TILE;
        const int key = it.key0 + r % TILE;
        if (key >= p.len_kv || c * 8 >= p.dim) continue;
        float4 x[PARTS][2];                     // all on their way before the first is used
#pragma unroll
        for (int i = 0; i < PARTS; ++i) x[i][0] = get_sums(at, DH, r, c, 0, i), x[i][1] = get_sums(at, DH, r, c, 1, i);
        float4 lo = x[0][0], hi = x[0][1];
#pragma unroll
        for (int i = 1; i < PARTS; ++i) {
            lo.x += x[i][0].x, lo.y += x[i][0].y, lo.z += x[i][0].z, lo.w += x[i][0].w;
            hi.x += x[i][1].x, hi.y += x[i][1].y, hi.z += x[i][1].z, hi.w += x[i][1].w;
        }
        const float by = dv ? 1.0f : p.scale;
        const int64_t *stride = dv ? p.dv_stride : p.dk_stride;
        *reinterpret_cast<uint4 *>((dv ? p.dv : p.dk) + it.b * stride[0] + key * stride[1] + it.h_kv * stride[2] + c * 8) =
            make_uint4(pack_bf16(lo.x * by, lo.y * by), pack_bf16(lo.z * by, lo.w * by), pack_bf16(hi.x * by, hi.y * by), pack_bf16(hi.z * by, hi.w * by));
    }
}

template <int DH, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
k_attn_backward(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                const __grid_constant__ CUtensorMap map_do, const AttnParams p) {
    extern __shared__ uint8_t raw[];
    using Dq = DqTiles<DH>;
    using Dkv = DkvTiles<DH>;
    using KeyItem = DkvItem<SPLIT>;
    constexpr uint32_t TILE_BYTES = Dq::TILE_BYTES;
    auto &sm = *reinterpret_cast<BwdSmem<DH> *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    BwdCommon &cm = sm.common;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, key_items = p.batch * p.heads_kv * p.tiles_kv, all_items = key_items + p.batch * p.heads * p.tiles_q;
    const int first_block = SPLIT ? blockIdx.x / p.parts : blockIdx.x;       // with SPLIT a key tile, or none

    if (threadIdx.x == 0) {
        queue_init(cm.queue, QUEUE_READERS);
        for (int i = 0; i < 2; ++i) {
            bar_init(&cm.dq.q_full[i], 1), bar_init(&cm.dq.q_free[i], 1), bar_init(&cm.dkv.kv_full[i], 1), bar_init(&cm.dkv.kv_free[i], 1);
            bar_init(&cm.dq.s_full[i], 1), bar_init(&cm.dq.dp_full[i], 1), bar_init(&cm.dq.ds_ready[i], 4), bar_init(&cm.dq.dq_done[i], 1);
            bar_init(&cm.dkv.s_full[i], 1), bar_init(&cm.dkv.dp_full[i], 1), bar_init(&cm.dkv.p_ready[i], 4), bar_init(&cm.dkv.ds_ready[i], 4);
            bar_init(&cm.dkv.dv_done[i], 1), bar_init(&cm.dkv.dk_done[i], 1);
        }
        for (int i = 0; i < DqBars::K_MOST; ++i) bar_init(&cm.dq.k_full[i], 1), bar_init(&cm.dq.k_free[i], 1);
        for (int i = 0; i < DqBars::V_MOST; ++i) bar_init(&cm.dq.v_full[i], 1), bar_init(&cm.dq.v_free[i], 1);
        for (int i = 0; i < DkvBars::Q_MOST; ++i) bar_init(&cm.dkv.q_full[i], 1), bar_init(&cm.dkv.q_free[i], 1);
        for (int i = 0; i < DkvBars::DO_MOST; ++i) bar_init(&cm.dkv.do_full[i], 1), bar_init(&cm.dkv.do_free[i], 1);
        bar_init(&cm.dq.s_taken, 4), bar_init(&cm.dq.dp_taken, 4), bar_init(&cm.dq.sums_full, 1), bar_init(&cm.dq.sums_taken, 8);
        bar_init(&cm.dkv.s_taken, Dkv::TURNS ? 4 : 8), bar_init(&cm.dkv.dp_taken, 4), bar_init(&cm.dkv.sums_full, 1), bar_init(&cm.dkv.sums_taken, 8);
        bar_init(&cm.landed, 1);
        cm.waits = {p.wait_ns, 0};
    }
    if (threadIdx.x < TILE && first_block < key_items) {
        constexpr uint32_t ONE = 0x3F80;                 // bf16
        sm.dkv.ones_lse[threadIdx.x] = make_uint4(ONE | ONE << 16, ONE, 0, 0);
        sm.dkv.ones_delta[threadIdx.x] = make_uint4(0, ONE << 16, ONE | ONE << 16, 0);
        sm.dkv.zeros[threadIdx.x] = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    if (warp == WARP_SCORES) tmem_alloc(&cm.tmem, TMEM_COLUMNS);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = cm.tmem;
    volatile Patience *waits = &cm.waits;
    after_previous();                           // k_attn_stats

    int block = first_block;                    // every role goes through the same items
    uint32_t items = 0, landed_phase = 0;       // answers read
    bool ok = true;
    const bool no_key_tile = SPLIT && first_block >= key_items;
    auto next = [&] { block = queue_next<true>(cm.queue, items++, waits), ok = ok && block >= 0; };
    auto next_one = [&] { block = queue_next_one<true>(cm.queue, items++, waits), ok = ok && block >= 0; };
    auto all_done = [&](const bool joins) {     // of the key tiles, in all roles
        fence_async_smem();
        tmem_fence_before();
        asm volatile("barrier.sync 1, %0;" ::"n"(THREADS) : "memory");
        if constexpr (SPLIT) {
            cluster_sync();
            if (joins && first_block < key_items) {
                if (p.parts == 2) join_sums<DH, 2>(p, first_block, smem_addr(&sm));
                else if (p.parts == 4) join_sums<DH, 4>(p, first_block, smem_addr(&sm));
                else join_sums<DH, 8>(p, first_block, smem_addr(&sm));
            }
            fence_async_smem();
            cluster_sync();                     // the others have read what is here
        }
        tmem_fence_after();
        if (waits->gave_up) ok = false;
    };
    auto ask = [&] {                            // once to an item, by the warp that brings the tiles
        if (!bar_wait(&cm.queue.free[items % QUEUE], (items / QUEUE + 1) & 1, waits)) return false;
        if (lane == 0) queue_count(cm.queue, items, p.next_item, SPLIT ? key_items : gridDim.x, all_items);
        __syncwarp();
        return true;
    };

    // dP, or the sums (with heads of up to 128 both, in the sums' thread), of the key tiles
    auto dkv_products = [&](const bool sums) {
        if (elected()) {
            DkvBars &bars = cm.dkv;
            const uint32_t zeros = smem_addr(sm.dkv.zeros), v_at = smem_addr(sm.dkv.v), q_at = smem_addr(sm.dkv.q), do_at = smem_addr(sm.dkv.dout), terms_at = smem_addr(sm.dkv.terms),
                           ones = smem_addr(sm.dkv.ones_delta);
            uint32_t sets = 0, tiles_in = 0;
            if (no_key_tile) next_one();
            auto dprobs = [&](uint32_t g, uint32_t set) {
                const uint32_t qs = g % Dkv::Q_SLOTS, ds = g % Dkv::DO_SLOTS;
                if (!bar_wait_one(&bars.q_full[qs], g / Dkv::Q_SLOTS & 1, waits)) return false;        // delta comes with the queries
                if (!bar_wait_one(&bars.do_full[ds], g / Dkv::DO_SLOTS & 1, waits)) return false;
                if (!Dkv::TURNS && !bar_wait_one(&bars.s_taken, g & 1, waits)) return false;
                if (Dkv::TURNS && g > 0 && !bar_wait_one(&bars.dp_taken, (g - 1) & 1, waits)) return false;
                tmem_fence_after();
                product_short<TILE>(tmem + Dkv::dprobs(g), ones, terms_at + qs * TILE * 16, zeros);
                product_rows<DH, TILE>(tmem + Dkv::dprobs(g), v_at + set * TILE_BYTES, do_at + ds * TILE_BYTES, true);
                mma_commit(&bars.dp_full[g & 1]);
                return true;
            };
            while (ok && block < key_items) {
                const KeyItem it(p, block);
                const uint32_t set = sets % Dkv::SETS;
                if (it.n > 0 && (sums || Dkv::TURNS)) {
                    ok = bar_wait_one(&bars.kv_full[set], sets / Dkv::SETS & 1, waits);
                    if (sums && sets > 0 && ok) ok = bar_wait_one(&bars.sums_taken, (sets - 1) & 1, waits);      // the last item's sums have been read
                    ++sets;
                }
                if (!sums) {
                    if (Dkv::TURNS)
                        for (int i = 0; ok && i < it.n; ++i) ok = dprobs(tiles_in + i, set);
                } else if (Dkv::TURNS) {
                    for (int i = 0; ok && i < it.n; ++i) {
                        const uint32_t g = tiles_in + i, qs = g % Dkv::Q_SLOTS, ds = g % Dkv::DO_SLOTS, w = g & 1;
                        ok = bar_wait_one(&bars.do_full[ds], g / Dkv::DO_SLOTS & 1, waits) && bar_wait_one(&bars.p_ready[w], g / 2 & 1, waits);
                        if (!ok) break;
                        tmem_fence_after();
                        product_down<DH, TILE>(tmem + Dkv::DV, tmem + Dkv::MINE + w * 64, do_at + ds * TILE_BYTES, i > 0);
                        mma_commit(&bars.dv_done[w]);
                        ok = bar_wait_one(&bars.q_full[qs], g / Dkv::Q_SLOTS & 1, waits) && bar_wait_one(&bars.ds_ready[w], g / 2 & 1, waits);
                        if (!ok) break;
                        tmem_fence_after();
                        product_down<DH, TILE>(tmem + Dkv::DK, tmem + Dkv::MINE + w * 64, q_at + qs * TILE_BYTES, i > 0);
                        mma_commit(&bars.dk_done[w]);
                        mma_commit(&bars.q_free[qs]);           // dS came from scores and dP: all products with the two tiles are done
                        mma_commit(&bars.do_free[ds]);
                    }
                } else if (it.n > 0 && ok) {
                    ok = dprobs(tiles_in, set);
                    for (int i = 0; ok && i < it.n; ++i) {
                        const uint32_t g = tiles_in + i, qs = g % Dkv::Q_SLOTS, ds = g % Dkv::DO_SLOTS;
                        for (int w = 0; w < 2 && ok; ++w) {     // each group's 64 queries; dK first: there is room for two query tiles only
                            ok = bar_wait_one(&bars.ds_ready[w], g & 1, waits);
                            if (!ok) break;
                            tmem_fence_after();
                            product_down<DH, 64>(tmem + Dkv::DK, tmem + Dkv::dprobs(g) + w * 64 + 32, q_at + qs * TILE_BYTES + w * 64 * 128, i > 0 || w > 0);
                        }
                        if (!ok) break;
                        mma_commit(&bars.q_free[qs]);
                        for (int w = 0; w < 2; ++w) product_down<DH, 64>(tmem + Dkv::DV, tmem + Dkv::dprobs(g) + w * 64, do_at + ds * TILE_BYTES + w * 64 * 128, i > 0 || w > 0);
                        mma_commit(&bars.do_free[ds]);
                        if (i + 1 < it.n) ok = dprobs(g + 1, set);
                    }
                }
                if (sums && it.n > 0 && ok) {
                    mma_commit(&bars.sums_full);
                    mma_commit(&bars.kv_free[set]);
                }
                tiles_in += it.n;
                if (ok) next_one();
            }
        }
        __syncwarp();
    };
    // scores, or dP, of the query tiles: products of one form
    auto dq_products = [&](const bool is_dp) {
        if (elected()) {
            // two products of the same form: scores from Q and K, dP from dO and V
            DqBars &bars = cm.dq;
            const uint32_t a_at = is_dp ? smem_addr(sm.dq.dout) : smem_addr(sm.dq.q), b_at = is_dp ? smem_addr(sm.dq.v) : smem_addr(sm.dq.k), slots = is_dp ? Dq::V_SLOTS : Dq::K_SLOTS;
            uint64_t *const full = is_dp ? bars.v_full : bars.k_full, *const taken = is_dp ? &bars.dp_taken : &bars.s_taken, *const done = is_dp ? bars.dp_full : bars.s_full;
            uint32_t sets = 0, tiles_in = 0;
            while (ok) {
                const DqItem it(p, block - key_items);
                const uint32_t set = sets % Dq::SETS;
                if (it.n > 0) ok = bar_wait_one(&bars.q_full[set], sets / Dq::SETS & 1, waits), ++sets;
                for (int j = 0; ok && j < it.n; ++j) {
                    const uint32_t g = tiles_in + j, slot = g % slots;
                    ok = bar_wait_one(&full[slot], g / slots & 1, waits) && (g == 0 || bar_wait_one(taken, (g - 1) & 1, waits));
                    if (!ok) break;
                    tmem_fence_after();
                    product_rows<DH, TILE>(tmem + (is_dp ? TILE : 0), a_at + set * TILE_BYTES, b_at + slot * TILE_BYTES);
                    mma_commit(&done[g & 1]);
                    if (is_dp) mma_commit(&bars.v_free[slot]);
                }
                tiles_in += it.n;
                if (ok) next_one();
            }
        }
        __syncwarp();
    };
    if (warp == WARP_LOAD) {
        registers_give<REGISTERS_HELP>();
        {
            DkvBars &bars = cm.dkv;
            uint32_t sets = 0, tiles_in = 0;        // counts over all items
            if (no_key_tile) {
                ok = ask();
                if (ok) next();
            }
            while (ok && block < key_items) {
                ok = ask();
                if (!ok) break;
                const KeyItem it(p, block);
                const Seq seq(p, it.b);
                if (it.n > 0) {
                    const uint32_t set = sets % Dkv::SETS;
                    if (!(ok = bar_wait(&bars.kv_free[set], (sets / Dkv::SETS + 1) & 1, waits))) break;
                    ++sets;
                    if (lane == 0) {
                        bar_expect(&bars.kv_full[set], 2 * TILE_BYTES);
                        for (int c = 0; c < DH / 64; ++c) {
                            copy_tile(smem_addr(sm.dkv.k[set]) + c * CHUNK, &map_k, &bars.kv_full[set], c * 64, it.key0, it.h_kv, it.b);
                            copy_tile(smem_addr(sm.dkv.v[set]) + c * CHUNK, &map_v, &bars.kv_full[set], c * 64, it.key0, it.h_kv, it.b);
                        }
                    }
                    __syncwarp();
                    for (int i = 0; ok && i < it.n; ++i) {
                        const uint32_t g = tiles_in + i, qs = g % Dkv::Q_SLOTS, ds = g % Dkv::DO_SLOTS;
                        const int h = it.h_kv * it.shared + (it.from + i) / it.per_head, tile = it.first + (it.from + i) % it.per_head;
                        if (!(ok = bar_wait(&bars.q_free[qs], (g / Dkv::Q_SLOTS + 1) & 1, waits))) break;
                        // the terms arrive at the queries' barrier: their bytes are announced without an arrival
                        if (lane == 0) {
                            asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(&bars.q_full[qs])), "r"(static_cast<uint32_t>(sizeof(sm.dkv.terms[0]))) : "memory");
                            copy_bytes(smem_addr(sm.dkv.terms[qs]), p.stats[(static_cast<int64_t>(it.b) * p.heads + h) * p.tiles_q + tile].terms, sizeof(sm.dkv.terms[0]), &bars.q_full[qs]);
                        }
                        __syncwarp();
                        ok = load_tile<DH, true>(smem_addr(sm.dkv.q[qs]), sm.dkv.q[qs], &map_q, &bars.q_full[qs], &cm.landed, landed_phase, tile * TILE, seq.n, p.len_q, h, it.b, waits) &&
                             bar_wait(&bars.do_free[ds], (g / Dkv::DO_SLOTS + 1) & 1, waits) &&
                             load_tile<DH, true>(smem_addr(sm.dkv.dout[ds]), sm.dkv.dout[ds], &map_do, &bars.do_full[ds], &cm.landed, landed_phase, tile * TILE, seq.n, p.len_q, h, it.b, waits);
                    }
                    tiles_in += it.n;
                }
                if (ok) next();
            }
        }
        // Query tiles next, whose data comes where that of the key tiles was: dQ.
        all_done(false);
        {
            DqBars &bars = cm.dq;
            uint32_t sets = 0, tiles_in = 0;
            while (ok) {
                ok = ask();
                if (!ok) break;
                const DqItem it(p, block - key_items);
                const Seq seq(p, it.b);
                if (it.n > 0) {
                    const uint32_t set = sets % Dq::SETS;
                    if (!(ok = bar_wait(&bars.q_free[set], (sets / Dq::SETS + 1) & 1, waits))) break;
                    ++sets;
                    if (lane == 0) {
                        bar_expect(&bars.q_full[set], 2 * TILE_BYTES);
                        for (int c = 0; c < DH / 64; ++c) {
                            copy_tile(smem_addr(sm.dq.q[set]) + c * CHUNK, &map_q, &bars.q_full[set], c * 64, it.row0, it.h, it.b);
                            copy_tile(smem_addr(sm.dq.dout[set]) + c * CHUNK, &map_do, &bars.q_full[set], c * 64, it.row0, it.h, it.b);
                        }
                    }
                    __syncwarp();
                    for (int j = 0; ok && j < it.n; ++j) {
                        const uint32_t g = tiles_in + j, ks = g % Dq::K_SLOTS, vs = g % Dq::V_SLOTS;
                        ok = bar_wait(&bars.k_free[ks], (g / Dq::K_SLOTS + 1) & 1, waits) &&
                             load_tile<DH, true>(smem_addr(sm.dq.k[ks]), sm.dq.k[ks], &map_k, &bars.k_full[ks], &cm.landed, landed_phase, j * TILE, seq.m, p.len_kv, it.h_kv, it.b, waits) &&
                             bar_wait(&bars.v_free[vs], (g / Dq::V_SLOTS + 1) & 1, waits) &&
                             load_tile<DH, true>(smem_addr(sm.dq.v[vs]), sm.dq.v[vs], &map_v, &bars.v_full[vs], &cm.landed, landed_phase, j * TILE, seq.m, p.len_kv, it.h_kv, it.b, waits);
                    }
                    tiles_in += it.n;
                }
                if (ok) next();
            }
        }
    } else if (warp == WARP_SCORES) {
        registers_give<REGISTERS_HELP>();
        {
            if (elected()) {
                DkvBars &bars = cm.dkv;
                const uint32_t zeros = smem_addr(sm.dkv.zeros), k_at = smem_addr(sm.dkv.k), q_at = smem_addr(sm.dkv.q), terms_at = smem_addr(sm.dkv.terms), ones = smem_addr(sm.dkv.ones_lse);
                uint32_t sets = 0, tiles_in = 0;
                if (no_key_tile) next_one();
                while (ok && block < key_items) {
                    const KeyItem it(p, block);
                    const uint32_t set = sets % Dkv::SETS;
                    if (it.n > 0) ok = bar_wait_one(&bars.kv_full[set], sets / Dkv::SETS & 1, waits), ++sets;
                    for (int i = 0; ok && i < it.n; ++i) {
                        const uint32_t g = tiles_in + i, qs = g % Dkv::Q_SLOTS;
                        ok = bar_wait_one(&bars.q_full[qs], g / Dkv::Q_SLOTS & 1, waits);
                        if (Dkv::TURNS && g > 0) ok = ok && bar_wait_one(&bars.s_taken, (g - 1) & 1, waits);
                        // the products that read P and dS of tile g - 2 have ended
                        if (!Dkv::TURNS && g > 1) ok = ok && bar_wait_one(&bars.do_free[(g - 2) % Dkv::DO_SLOTS], (g - 2) / Dkv::DO_SLOTS & 1, waits);
                        if (!ok) break;
                        tmem_fence_after();
                        product_short<TILE>(tmem + Dkv::scores(g), ones, terms_at + qs * TILE * 16, zeros);
                        product_rows<DH, TILE>(tmem + Dkv::scores(g), k_at + set * TILE_BYTES, q_at + qs * TILE_BYTES, true);
                        mma_commit(&bars.s_full[g & 1]);
                    }
                    tiles_in += it.n;
                    if (ok) next_one();
                }
            }
            __syncwarp();
        }
        // Query tiles next, whose data comes where that of the key tiles was: dQ.
        all_done(false);
        dq_products(false);
    } else if (warp == WARP_DP) {
        registers_give<REGISTERS_HELP>();
        dkv_products(false);
        // Query tiles next, whose data comes where that of the key tiles was: dQ.
        all_done(false);
        dq_products(true);
    } else if (warp == WARP_SUMS) {
        registers_give<REGISTERS_HELP>();
        dkv_products(true);
        // Query tiles next, whose data comes where that of the key tiles was: dQ.
        all_done(false);
        {
            if (elected()) {
                DqBars &bars = cm.dq;
                const uint32_t k_at = smem_addr(sm.dq.k);
                uint32_t sets = 0, tiles_in = 0;
                while (ok) {
                    const DqItem it(p, block - key_items);
                    if (it.n > 0 && sets > 0) ok = bar_wait_one(&bars.sums_taken, (sets - 1) & 1, waits);      // the last item's sums have been read
                    for (int j = 0; ok && j < it.n; ++j) {
                        const uint32_t g = tiles_in + j, ks = g % Dq::K_SLOTS;
                        ok = bar_wait_one(&bars.k_full[ks], g / Dq::K_SLOTS & 1, waits) && bar_wait_one(&bars.ds_ready[g & 1], g / 2 & 1, waits);
                        if (!ok) break;
                        tmem_fence_after();
                        product_down<DH, TILE>(tmem + 3 * TILE, tmem + 2 * TILE + (g & 1) * 64, k_at + ks * TILE_BYTES, j > 0);
                        mma_commit(&bars.dq_done[g & 1]);
                        mma_commit(&bars.k_free[ks]);                // dS came from the scores: that product is done as well
                    }
                    if (it.n > 0 && ok) {
                        mma_commit(&bars.sums_full);
                        mma_commit(&bars.q_free[sets % Dq::SETS]);
                        ++sets;
                    }
                    tiles_in += it.n;
                    if (ok) next_one();
                }
            }
            __syncwarp();
        }
    } else {
        registers_take<REGISTERS_COMPUTE>();
        {
            DkvBars &bars = cm.dkv;
            constexpr int WIDTH = Dkv::TURNS ? TILE : TILE / 2, EVERY = Dkv::TURNS ? 2 : 1;      // columns of a tile that a group takes, of every EVERYth tile
            const int w = warp / 4, col0 = Dkv::TURNS ? 0 : w * WIDTH;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16);
            uint32_t tiles_in = 0, outputs = 0;
            if (no_key_tile) next();
            while (ok && block < key_items) {
                const KeyItem it(p, block);
                const Seq seq(p, it.b);
                const int key = it.key0 + threadIdx.x % TILE;
                int i = Dkv::TURNS ? static_cast<int>((tiles_in + w) & 1) : 0, column = it.from + i;             // query tile of its head
                for (; i < it.n; i += EVERY, column += EVERY) {
                    const uint32_t g = tiles_in + i;
                    // Tiles in turn have barriers in turn: a group that waited for one of them only every other time would
                    // tell its phases apart by nothing.
                    uint64_t *const s_full = &bars.s_full[g & 1], *const dp_full = &bars.dp_full[g & 1];
                    const uint32_t s_at = lanes + Dkv::scores(g) + col0, dp_at = lanes + Dkv::dprobs(g) + col0;
                    const uint32_t p_at = Dkv::TURNS ? lanes + Dkv::MINE + w * 64 : dp_at, ds_at = Dkv::TURNS ? p_at : dp_at + 32;
                    while (column >= it.per_head) column -= it.per_head;
                    const int row0 = (it.first + column) * TILE;
                    // columns before `hidden` do not see the key
                    const int hidden = seq.causal && row0 < it.key0 + TILE - 1 - seq.shift ? key - seq.shift - row0 - col0 : 0;
                    if (!(ok = bar_wait(s_full, g / 2 & 1, waits))) break;
                    tmem_fence_after();
                    uint32_t s[WIDTH / 32][32], probs[WIDTH / 64][32];
#pragma unroll
                    for (int q = 0; q < WIDTH / 32; ++q) tmem_load32(s_at + q * 32, s[q]);
                    tmem_wait_loads(s);
                    tmem_fence_before();
                    bar_arrive_warp(&bars.s_taken);
                    if (__any_sync(0xFFFFFFFFu, hidden > 0)) {
#pragma unroll
                        for (int c = 0; c < WIDTH; ++c)
                            if (c < hidden) s[c / 32][c % 32] = __float_as_uint(-INFINITY);
                    }
#pragma unroll
                    for (int c = 0; c < WIDTH; c += 2) {
                        const float2 x = mul2(pair_of(s[c / 32], c % 32), both(p.scale_log2));
                        const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
                        s[c / 32][c % 32] = __float_as_uint(e.x), s[c / 32][c % 32 + 1] = __float_as_uint(e.y);
                        probs[c / 64][c % 64 / 2] = pack_bf16(e);
                    }
                    if constexpr (Dkv::TURNS) {
                        if (g > 1) {                         // its last dS has been used
                            if (!(ok = bar_wait(&bars.dk_done[w], (g / 2 - 1) & 1, waits))) break;
                            tmem_fence_after();
                        }
                        tmem_store32(p_at, probs[0]);
                        tmem_store32(p_at + 32, probs[WIDTH / 64 - 1]);
                        tmem_wait_stores();
                        tmem_fence_before();
                        bar_arrive_warp(&bars.p_ready[w]);
                    }
                    if (!(ok = bar_wait(dp_full, g / 2 & 1, waits))) break;
                    tmem_fence_after();
                    uint32_t d[2][32];
                    if constexpr (Dkv::TURNS) {
                        uint32_t packed[4][16];
                        tmem_load32(dp_at, d[0]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {        // while 32 columns are worked on, the next are on their way
                            tmem_wait_loads(d[q % 2]);
                            if (q < 3) {
                                tmem_load32(dp_at + (q + 1) * 32, d[(q + 1) % 2]);
                            } else {
                                tmem_fence_before();
                                bar_arrive_warp(&bars.dp_taken);
                            }
#pragma unroll
                            for (int c = 0; c < 32; c += 2) packed[q][c / 2] = pack_bf16(mul2(pair_of(s[q], c), pair_of(d[q % 2], c)));
                        }
                        if (!(ok = bar_wait(&bars.dv_done[w], g / 2 & 1, waits))) break;        // P has been used
                        tmem_fence_after();
#pragma unroll
                        for (int q = 0; q < 4; ++q) tmem_store16(ds_at + q * 16, packed[q]);
                    } else {
                        tmem_load32(dp_at, d[0]);
                        tmem_load32(dp_at + 32, d[1]);
                        tmem_wait_loads(d);
                        tmem_store32(p_at, probs[0]);
                        uint32_t packed[32];
#pragma unroll
                        for (int c = 0; c < 64; c += 2) packed[c / 2] = pack_bf16(mul2(pair_of(s[c / 32], c % 32), pair_of(d[c / 32], c % 32)));
                        tmem_store32(ds_at, packed);
                    }
                    tmem_wait_stores();
                    tmem_fence_before();
                    bar_arrive_warp(&bars.ds_ready[w]);
                }
                if (!ok) break;
                tiles_in += it.n;
                if constexpr (SPLIT) {               // all products that read the tiles are done with the sums
                    if (it.n > 0) ok = bar_wait(&bars.sums_full, 0, waits);
                    tmem_fence_after();
#pragma unroll
                    for (int c = 0; c < DH; c += 32) {
                        uint32_t o[32];
                        tmem_load32(lanes + (w == 0 ? Dkv::DV : Dkv::DK) + c, o);
                        tmem_wait_loads(o);
                        put_sums(&sm, DH, threadIdx.x, c, o, it.n == 0 || key >= seq.m);
                    }
                    if (ok) next();
                    continue;
                }
                // one group writes dV, the other dK
                const int64_t *stride = w == 0 ? p.dv_stride : p.dk_stride;
                __nv_bfloat16 *out = (w == 0 ? p.dv : p.dk) + it.b * stride[0] + key * stride[1] + it.h_kv * stride[2];
                if (it.n > 0) {
                    if (!(ok = bar_wait(&bars.sums_full, outputs & 1, waits))) break;
                    ++outputs;
                    tmem_fence_after();
#pragma unroll
                    for (int c = 0; c < DH; c += 64) {
                        uint32_t o[2][32];
                        tmem_load32(lanes + (w == 0 ? Dkv::DV : Dkv::DK) + c, o[0]);
                        tmem_load32(lanes + (w == 0 ? Dkv::DV : Dkv::DK) + c + 32, o[1]);
                        tmem_wait_loads(o);
                        if (c == DH - 64) {
                            tmem_fence_before();
                            bar_arrive_warp(&bars.sums_taken);
                        }
                        if (key >= seq.m)
#pragma unroll
                            for (int e = 0; e < 64; ++e) o[e / 32][e % 32] = 0;
                        const float by = w == 0 ? 1.0f : p.scale;
                        if (key < p.len_kv) write_columns(out, c, p.dim, o[0], by), write_columns(out, c + 32, p.dim, o[1], by);
                    }
                } else if (key < p.len_kv) {
                    write_zeros(out, 0, p.dim);
                }
                next();
            }
        }
        // Query tiles next, whose data comes where that of the key tiles was: dQ.
        all_done(true);
        {
            DqBars &bars = cm.dq;
            const int w = warp / 4, in_tile = threadIdx.x % TILE;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16), s_at = lanes, dp_at = lanes + TILE, ds_at = lanes + 2 * TILE + w * 64;
            uint32_t tiles_in = 0, outputs = 0;
            while (ok) {
                const DqItem it(p, block - key_items);
                const Seq seq(p, it.b);
                const int row = it.row0 + in_tile, limit = seq.keys_of(row), all_see = seq.keys_of(it.row0);
                const bool whole = it.row0 + TILE <= seq.n;
                const QueryStats &stats = p.stats[static_cast<int64_t>(it.bh) * p.tiles_q + it.tile];
                const float lse = stats.lse[in_tile], delta = stats.delta[in_tile];
                for (int j = static_cast<int>((tiles_in + w) & 1); j < it.n; j += 2) {
                    const uint32_t g = tiles_in + j;
                    if (!(ok = bar_wait(&bars.s_full[w], g / 2 & 1, waits))) break;
                    tmem_fence_after();
                    uint32_t s[4][32];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_load32(s_at + q * 32, s[q]);
                    tmem_wait_loads(s);
                    tmem_fence_before();
                    bar_arrive_warp(&bars.s_taken);
                    if (!whole || (j + 1) * TILE > all_see) {
                        const int left = limit - j * TILE;           // columns that the row sees
#pragma unroll
                        for (int c = 0; c < TILE; ++c)
                            if (c >= left) s[c / 32][c % 32] = __float_as_uint(-INFINITY);
                    }
#pragma unroll
                    for (int c = 0; c < TILE; c += 2) {
                        const float2 x = fma2(pair_of(s[c / 32], c % 32), both(p.scale_log2), both(-lse));
                        s[c / 32][c % 32] = __float_as_uint(exp2_fast(x.x)), s[c / 32][c % 32 + 1] = __float_as_uint(exp2_fast(x.y));
                    }
                    if (!(ok = bar_wait(&bars.dp_full[w], g / 2 & 1, waits))) break;
                    tmem_fence_after();
                    uint32_t d[2][32], packed[4][16];
                    tmem_load32(dp_at, d[0]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {        // while 32 columns are worked on, the next are on their way
                        tmem_wait_loads(d[q % 2]);
                        if (q < 3) {
                            tmem_load32(dp_at + (q + 1) * 32, d[(q + 1) % 2]);
                        } else {
                            tmem_fence_before();
                            bar_arrive_warp(&bars.dp_taken);
                        }
#pragma unroll
                        for (int c = 0; c < 32; c += 2) packed[q][c / 2] = pack_bf16(mul2(pair_of(s[q], c), add2(pair_of(d[q % 2], c), both(-delta))));
                    }
                    if (g > 1) {                         // its last dS has been used
                        if (!(ok = bar_wait(&bars.dq_done[w], (g / 2 - 1) & 1, waits))) break;
                        tmem_fence_after();
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_store16(ds_at + q * 16, packed[q]);
                    tmem_wait_stores();
                    tmem_fence_before();
                    bar_arrive_warp(&bars.ds_ready[w]);
                }
                if (!ok) break;
                tiles_in += it.n;
                __nv_bfloat16 *out = p.out + it.b * p.out_stride[0] + row * p.out_stride[1] + it.h * p.out_stride[2];
                if (it.n > 0) {
                    if (!(ok = bar_wait(&bars.sums_full, outputs & 1, waits))) break;
                    ++outputs;
                    tmem_fence_after();
                    uint32_t o[DH / 64][32];                 // a group writes half of the columns
#pragma unroll
                    for (int c = 0; c < DH / 64; ++c) tmem_load32(lanes + 3 * TILE + w * (DH / 2) + c * 32, o[c]);
                    tmem_wait_loads(o);
                    tmem_fence_before();
                    bar_arrive_warp(&bars.sums_taken);
#pragma unroll
                    for (int c = 0; c < DH / 64; ++c) {
                        if (limit == 0)
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[c][e] = 0;
                        if (row < p.len_q) write_columns(out, w * (DH / 2) + c * 32, p.dim, o[c], p.scale);
                    }
                } else if (row < p.len_q) {
                    write_zeros(out, w * (DH / 2), min((w + 1) * (DH / 2), p.dim));
                }
                next();
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (waits->gave_up) {
        settle();
        if (warp < 8) {
            fill_nan(p.out, p.out_stride, p.batch, p.len_q, p.heads, p.dim);
            fill_nan(p.dk, p.dk_stride, p.batch, p.len_kv, p.heads_kv, p.dim);
            fill_nan(p.dv, p.dv_stride, p.batch, p.len_kv, p.heads_kv, p.dim);
        }
    }
    if (warp == WARP_SCORES) tmem_free(tmem, TMEM_COLUMNS);
}

// ---------------------------------------------------------------------------------- host side
int make_map(CUtensorMap *map, const char *what, const void *at, const int64_t *stride, int batch, int tokens, int heads, int dim) {
    const encode_fn encode = encoder();
    if (encode == nullptr) return fail(KT_ERR_CUDA, "the driver does not offer cuTensorMapEncodeTiled");
    const cuuint64_t sizes[4] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(tokens), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(batch)};
    // the stride of a dimension of one is never used
    const cuuint64_t strides[3] = {tokens > 1 ? static_cast<cuuint64_t>(stride[1]) * 2 : 16, heads > 1 ? static_cast<cuuint64_t>(stride[2]) * 2 : 16,
                                   batch > 1 ? static_cast<cuuint64_t>(stride[0]) * 2 : 16};
    const cuuint32_t box[4] = {64, TILE, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult rc = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(at), sizes, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc != CUDA_SUCCESS) return fail(KT_ERR_CUDA, "describing %s to the copy engine failed with driver status %d", what, static_cast<int>(rc));
    return KT_OK;
}

// `written`: an output, no two rows of which may share elements (the bits would depend on who writes last): each
// stride, in rising order, clears what those before it span.
int check_heads(const char *what, const void *at, const int64_t *stride, int batch, int tokens, int heads, int dim, bool written) {
    if (at == nullptr) return fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(at) % 16) return fail(KT_ERR_ALIGN, "%s is not 16-byte aligned", what);
    const int size[3] = {batch, tokens, heads};
    for (int i = 0; i < 3; ++i) {
        if (size[i] <= 1) continue;
        if (stride[i] % 8) return fail(KT_ERR_ALIGN, "%s: the strides of batch, token and head must be multiples of 8 elements", what);
        if (stride[i] < 8 || stride[i] >= INT64_C(1) << 38) return fail(KT_ERR_SHAPE, "%s: a stride of %lld elements (expanded tensors need a copy)", what, (long long)stride[i]);
    }
    if (!written) return KT_OK;
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    __int128 span = dim;                        // (2^30 steps of 2^38 elements, three times)
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (stride[i] < span) return fail(KT_ERR_SHAPE, "%s: tokens, heads or sequences of an output overlap (a stride of %lld elements)", what, (long long)stride[i]);
        span += static_cast<__int128>(stride[i]) * (size[i] - 1);
    }
    return KT_OK;
}

std::atomic<int64_t> wait_limit{2000000000};     // of all kernels that wait

int fill(const kt_attn *a, AttnParams *p) {
    if (a == nullptr) return fail(KT_ERR_INVALID, "the description is NULL");
    if (a->dtype != KT_BF16) return fail(KT_ERR_INVALID, "attention takes KT_BF16 heads");
    if (a->batch < 0 || a->len_q < 0 || a->len_kv < 0 || a->heads < 1 || a->heads_kv < 1) return fail(KT_ERR_SHAPE, "negative sizes or no heads");
    if (a->heads % a->heads_kv) return fail(KT_ERR_SHAPE, "%d query heads cannot share %d key/value heads", a->heads, a->heads_kv);
    if (a->head_dim < 8 || a->head_dim > KT_ATTN_MAX_DIM || a->head_dim % 8) return fail(KT_ERR_SHAPE, "head_dim %d: a multiple of 8 up to %d expected", a->head_dim, KT_ATTN_MAX_DIM);
    if (!(a->scale >= 1.0f / (1 << 20)) || !(a->scale <= 1 << 20)) return fail(KT_ERR_INVALID, "scale must be from 2^-20 to 2^20");
    if (a->len_q > (1 << 30) || a->len_kv > (1 << 30)) return fail(KT_ERR_SHAPE, "more than 2^30 tokens");
    *p = AttnParams{};
    p->batch = a->batch, p->heads = a->heads, p->heads_kv = a->heads_kv, p->len_q = a->len_q, p->len_kv = a->len_kv, p->dim = a->head_dim;
    p->causal = a->causal != 0, p->used_q = a->used_q, p->used_kv = a->used_kv, p->scale = a->scale, p->scale_log2 = a->scale * LOG2E, p->wait_ns = static_cast<uint64_t>(wait_limit.load(std::memory_order_relaxed));
    p->tiles_q = (p->len_q + TILE - 1) / TILE, p->tiles_kv = (p->len_kv + TILE - 1) / TILE;
    if (static_cast<int64_t>(p->batch) * p->heads * (p->tiles_q > p->tiles_kv ? p->tiles_q : p->tiles_kv) > INT64_C(1) << 27)
        return fail(KT_ERR_SHAPE, "batch x heads x tokens is too large");
    for (const int32_t *u : {a->used_q, a->used_kv})
        if (reinterpret_cast<uintptr_t>(u) % 4) return fail(KT_ERR_ALIGN, "used_q or used_kv is not 4-byte aligned");
    return KT_OK;
}

template <typename Smem, auto KERNEL>
int room(size_t *bytes) {
    static std::atomic<uint64_t> raised{0};      // a bit for each device on which the kernel's limit has been raised
    *bytes = sizeof(Smem) + 1024;                // the tiles start at a multiple of 1024
    int dev = 0;
    KT_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
        KT_CUDA(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(*bytes)));
        raised.fetch_or(bit, std::memory_order_relaxed);
    }
    return KT_OK;
}

// CTAs to a work item of the forward pass (1, 2, 4 or 8): few long items leave SMs without work, yet a CTA of a split
// item costs its start, which nothing overlaps, and the join.  Estimated in steps of one key tile (some 1.6 us),
// from the sizes alone, with the figures of the join fitted to these times in us (1, 2, 4, 8 CTAs):
//   1 query, 8192 keys, 8 heads of 128          97   52   31   20
//   2048 queries and keys, 8 heads of 64        31   23   35   75
//   2 x 6499 causal, 2 heads of 64              80   48   73  124
//   2 x 4096, 8 heads of 64 (256 items)        103  129  176  310
int parts_of(const AttnParams &p) {
    const int64_t pairs = (p.tiles_q + 1) / 2, all = static_cast<int64_t>(p.batch) * p.heads, items = pairs * all;
    if (items > 4 * SMS) return 1;
    int64_t longest = 0, sum = 0;
    for (int64_t i = 0; i < pairs; ++i) {
        const int64_t last = (i + 1) * 2 * TILE < p.len_q ? (i + 1) * 2 * TILE : p.len_q, seen = last + p.len_kv - p.len_q;
        const int64_t n = !p.causal ? p.tiles_kv : seen > 0 ? (seen + TILE - 1) / TILE : 0;
        sum += n, longest = n > longest ? n : longest;
    }
    const double mean = static_cast<double>(sum) / pairs, rows = p.len_q < 2 * TILE ? p.len_q : 2 * TILE;
    int best = 1;
    double least = 0.0;
    for (int parts = 1; parts <= 8; parts *= 2) {
        const double each = parts == 1 ? 0.0 : 4.0 + parts * rows / (2 * TILE), rounds = static_cast<double>((items * parts + SMS - 1) / SMS);
        const double all_rounds = rounds * (mean / parts + each), one = static_cast<double>(longest) / parts + each;
        const double cost = (all_rounds > one ? all_rounds : one) + (parts == 1 ? 3.0 : 0.0);
        if (parts == 1 || cost < least) best = parts, least = cost;
    }
    return best;
}

template <int DH>
int start_forward(const CUtensorMap (&m)[3], AttnParams &p, cudaStream_t st) {
    size_t bytes = 0;
    p.parts = parts_of(p);
    const unsigned grid = static_cast<unsigned>(p.batch * p.heads * ((p.tiles_q + 1) / 2) * p.parts);
    if (p.parts == 1) {
        if (int rc = room<FwdSmem<DH>, k_attn_forward<DH, false>>(&bytes)) return rc;
        k_attn_forward<DH, false><<<grid, THREADS, bytes, st>>>(m[0], m[1], m[2], p);
        KT_CUDA(cudaGetLastError());
        return KT_OK;
    }
    if (int rc = room<FwdSmem<DH>, k_attn_forward<DH, true>>(&bytes)) return rc;
    KT_CUDA(launch_joint(k_attn_forward<DH, true>, p.parts, dim3(grid), dim3(THREADS), bytes, st, m[0], m[1], m[2], p));
    return KT_OK;
}

// CTAs that share a key tile in the backward pass (1, 2, 4 or 8).  Key tiles that many queries see, of many heads, are
// long, and where they are few the longest decides.  Estimated in steps of one query tile, from the sizes alone: the
// longest key tile, or all work over all SMs; a share costs some 5 + parts steps besides, for the join and the
// wait for it.  Measured in us with 1, 2, 4 and 8:
//   2048 causal, 8 heads of 128 on 1           185   125    85    67      (16 key tiles, 128 steps the longest)
//   4 x 700 causal, 8 heads of 128 on 1         91    60    47            (24, 48 steps)
//   4096 queries on 77 keys, 8 heads of 64      48    34    28    26      (8, 32 steps)
//   2 x 578 causal, 4 heads of 64 on 2          20    19    25            (20, 10 steps)
int parts_of_keys(const AttnParams &p) {
    const int64_t all = static_cast<int64_t>(p.batch) * p.heads_kv, key_tiles = all * p.tiles_kv, gap = p.len_kv - p.len_q;
    if (key_tiles * 2 > SMS) return 1;
    int64_t longest = 0, sum = 0;
    for (int64_t i = 0; i < p.tiles_kv; ++i) {
        const int64_t unseen = p.causal && i * TILE > gap ? (i * TILE - gap) / TILE : 0, n = unseen < p.tiles_q ? (p.tiles_q - unseen) * (p.heads / p.heads_kv) : 0;
        sum += n, longest = n > longest ? n : longest;
    }
    const double busy = 1.5 * (sum * all) / SMS;          // a step of a query tile is half of one of a key tile
    int best = 1;
    double least = 0.0;
    for (int parts = 1; parts <= 8 && key_tiles * parts <= (parts < 8 ? SMS : 128); parts *= 2) {      // 16 clusters of 8 have a place at once
        const double each = static_cast<double>(longest) / parts, cost = (each > busy ? each : busy) + (parts > 1 ? 5 + parts : 0);
        if (parts == 1 || cost < least) best = parts, least = cost;
    }
    return best;
}

template <int DH>
int start_backward(const CUtensorMap (&m)[4], AttnParams &p, cudaStream_t st) {
    size_t bytes = 0;
    const int items = p.batch * (p.heads_kv * p.tiles_kv + p.heads * p.tiles_q);
    p.parts = parts_of_keys(p);
    if (p.parts > 1) {
        if (int rc = room<BwdSmem<DH>, k_attn_backward<DH, true>>(&bytes)) return rc;
        const int key_ctas = p.batch * p.heads_kv * p.tiles_kv * p.parts, useful = key_ctas + p.batch * p.heads * p.tiles_q;
        const int grid = (useful < SMS ? useful : SMS) / p.parts * p.parts;       // key_ctas at least: parts_of_keys
        KT_CUDA(launch_behind(k_attn_backward<DH, true>, p.parts, dim3(grid), dim3(THREADS), bytes, st, m[0], m[1], m[2], m[3], p));
        return KT_OK;
    }
    if (int rc = room<BwdSmem<DH>, k_attn_backward<DH, false>>(&bytes)) return rc;
    KT_CUDA(launch_behind(k_attn_backward<DH, false>, 1, dim3(items < SMS ? items : SMS), dim3(THREADS), bytes, st, m[0], m[1], m[2], m[3], p));
    return KT_OK;
}

// Rows of zeros where there is nothing to attend to (no keys at all).
int clear(__nv_bfloat16 *at, const int64_t *stride, int batch, int tokens, int heads, int dim, cudaStream_t st) {
    for (int b = 0; b < batch; ++b)
        for (int h = 0; h < heads; ++h)
            KT_CUDA(cudaMemset2DAsync(at + b * stride[0] + h * stride[2], static_cast<size_t>(tokens > 1 ? stride[1] : dim) * 2, 0, static_cast<size_t>(dim) * 2, tokens, st));
    return KT_OK;
}

void copy_strides(int64_t *to, const int64_t *from) {
    for (int i = 0; i < 3; ++i) to[i] = from[i];
}

}  // namespace

uint64_t ktd::wait_limit_ns() { return static_cast<uint64_t>(wait_limit.load(std::memory_order_relaxed)); }

extern "C" {

int kt_attn_forward(const kt_attn *a, const void *q, const int64_t *q_stride, const void *k, const int64_t *k_stride, const void *v,
                    const int64_t *v_stride, void *out, const int64_t *out_stride, float *lse, void *stream) {
    AttnParams p;
    if (int rc = fill(a, &p)) return rc;
    if (p.batch == 0 || p.len_q == 0) return KT_OK;
    if (!q_stride || !k_stride || !v_stride || !out_stride) return fail(KT_ERR_INVALID, "a stride array is NULL");
    if (int rc = check_heads("q", q, q_stride, p.batch, p.len_q, p.heads, p.dim, false)) return rc;
    if (int rc = check_heads("out", out, out_stride, p.batch, p.len_q, p.heads, p.dim, true)) return rc;
    if (p.len_kv > 0) {
        if (int rc = check_heads("k", k, k_stride, p.batch, p.len_kv, p.heads_kv, p.dim, false)) return rc;
        if (int rc = check_heads("v", v, v_stride, p.batch, p.len_kv, p.heads_kv, p.dim, false)) return rc;
    }
    if (lse == nullptr) return fail(KT_ERR_INVALID, "lse is NULL");
    if (reinterpret_cast<uintptr_t>(lse) % 4) return fail(KT_ERR_ALIGN, "lse is not 4-byte aligned");
    p.out = static_cast<__nv_bfloat16 *>(out), p.lse = lse;
    copy_strides(p.out_stride, out_stride);
    CUtensorMap m[3];
    if (int rc = make_map(&m[0], "q", q, q_stride, p.batch, p.len_q, p.heads, p.dim)) return rc;
    // without keys the kernel copies nothing and only writes its empty rows: any valid map will do
    const bool keys = p.len_kv > 0;
    if (int rc = make_map(&m[1], "k", keys ? k : q, keys ? k_stride : q_stride, p.batch, keys ? p.len_kv : p.len_q, keys ? p.heads_kv : p.heads, p.dim)) return rc;
    if (int rc = make_map(&m[2], "v", keys ? v : q, keys ? v_stride : q_stride, p.batch, keys ? p.len_kv : p.len_q, keys ? p.heads_kv : p.heads, p.dim)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return p.dim <= 64 ? start_forward<64>(m, p, st) : start_forward<128>(m, p, st);
}

int64_t kt_attn_workspace(int batch, int heads, int len_q) {
    if (batch < 0 || heads < 0 || len_q < 0) return 0;
    return static_cast<int64_t>(batch) * heads * ((static_cast<int64_t>(len_q) + TILE - 1) / TILE) * static_cast<int64_t>(sizeof(QueryStats)) + 16;      // and the counter of items
}

int kt_attn_backward(const kt_attn *a, const void *dout, const int64_t *dout_stride, const void *q, const int64_t *q_stride, const void *k,
                     const int64_t *k_stride, const void *v, const int64_t *v_stride, const void *out, const int64_t *out_stride, const float *lse,
                     void *dq, const int64_t *dq_stride, void *dk, const int64_t *dk_stride, void *dv, const int64_t *dv_stride, void *workspace,
                     int64_t workspace_bytes, void *stream) {
    AttnParams p;
    if (int rc = fill(a, &p)) return rc;
    if (p.batch == 0 || (p.len_q == 0 && p.len_kv == 0)) return KT_OK;
    if (!dout_stride || !q_stride || !k_stride || !v_stride || !out_stride || !dq_stride || !dk_stride || !dv_stride) return fail(KT_ERR_INVALID, "a stride array is NULL");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    struct {
        const char *what;
        const void *at;
        const int64_t *stride;
        int tokens, heads;
        bool written;
    } const all[] = {{"dout", dout, dout_stride, p.len_q, p.heads, false}, {"q", q, q_stride, p.len_q, p.heads, false}, {"out", out, out_stride, p.len_q, p.heads, false},
                     {"dq", dq, dq_stride, p.len_q, p.heads, true}, {"k", k, k_stride, p.len_kv, p.heads_kv, false}, {"v", v, v_stride, p.len_kv, p.heads_kv, false},
                     {"dk", dk, dk_stride, p.len_kv, p.heads_kv, true}, {"dv", dv, dv_stride, p.len_kv, p.heads_kv, true}};
    for (const auto &t : all)
        if (t.tokens > 0)
            if (int rc = check_heads(t.what, t.at, t.stride, p.batch, t.tokens, t.heads, p.dim, t.written)) return rc;
    if (p.len_kv == 0) return clear(static_cast<__nv_bfloat16 *>(dq), dq_stride, p.batch, p.len_q, p.heads, p.dim, st);
    if (p.len_q == 0) {
        if (int rc = clear(static_cast<__nv_bfloat16 *>(dk), dk_stride, p.batch, p.len_kv, p.heads_kv, p.dim, st)) return rc;
        return clear(static_cast<__nv_bfloat16 *>(dv), dv_stride, p.batch, p.len_kv, p.heads_kv, p.dim, st);
    }
    if (lse == nullptr) return fail(KT_ERR_INVALID, "lse is NULL");
    if (reinterpret_cast<uintptr_t>(lse) % 4) return fail(KT_ERR_ALIGN, "lse is not 4-byte aligned");
    const int64_t need = kt_attn_workspace(p.batch, p.heads, p.len_q);
    if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
    if (workspace_bytes < need) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)workspace_bytes, (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
    CUtensorMap m[4];
    if (int rc = make_map(&m[0], "q", q, q_stride, p.batch, p.len_q, p.heads, p.dim)) return rc;
    if (int rc = make_map(&m[1], "k", k, k_stride, p.batch, p.len_kv, p.heads_kv, p.dim)) return rc;
    if (int rc = make_map(&m[2], "v", v, v_stride, p.batch, p.len_kv, p.heads_kv, p.dim)) return rc;
    if (int rc = make_map(&m[3], "dout", dout, dout_stride, p.batch, p.len_q, p.heads, p.dim)) return rc;
    p.o = static_cast<const __nv_bfloat16 *>(out), p.dout = static_cast<const __nv_bfloat16 *>(dout), p.lse = const_cast<float *>(lse), p.stats = static_cast<QueryStats *>(workspace);
    p.next_item = reinterpret_cast<unsigned *>(static_cast<char *>(workspace) + need - 16);
    copy_strides(p.o_stride, out_stride);
    copy_strides(p.dout_stride, dout_stride);
    const unsigned tiles_of_all = static_cast<unsigned>(p.batch * p.heads * p.tiles_q);
    p.dim <= 64 ? k_attn_stats<8><<<tiles_of_all, 256, 0, st>>>(p) : k_attn_stats<16><<<tiles_of_all, 256, 0, st>>>(p);
    KT_CUDA(cudaGetLastError());
    p.out = static_cast<__nv_bfloat16 *>(dq), p.dk = static_cast<__nv_bfloat16 *>(dk), p.dv = static_cast<__nv_bfloat16 *>(dv);
    copy_strides(p.out_stride, dq_stride);
    copy_strides(p.dk_stride, dk_stride);
    copy_strides(p.dv_stride, dv_stride);
    return p.dim <= 64 ? start_backward<64>(m, p, st) : start_backward<128>(m, p, st);
}

int kt_attn_wait_limit(int64_t nanoseconds) {
    if (nanoseconds < 0 || nanoseconds > INT64_C(60000000000)) return fail(KT_ERR_INVALID, "a limit of %lld ns: 0 to 60 s expected", (long long)nanoseconds);
    wait_limit.store(nanoseconds, std::memory_order_relaxed);
    return KT_OK;
}

int kt_attn_given_up(int64_t *count) {
    if (count == nullptr) return fail(KT_ERR_INVALID, "count is NULL");
    unsigned long long n = 0;
    KT_CUDA(cudaDeviceSynchronize());           // the copy alone waits for no stream that does not block
    KT_CUDA(cudaMemcpyFromSymbol(&n, g_waits_given_up, sizeof(n)));
    *count = static_cast<int64_t>(n);
    return KT_OK;
}

int kt_waits_given_up(int64_t *count) {
    if (int rc = kt_attn_given_up(count)) return rc;
    unsigned long long n = 0;
    for (auto of : {xent_given_up, orth_given_up}) {
        if (int rc = of(&n)) return rc;
        *count += static_cast<int64_t>(n);
    }
    return KT_OK;
}

}  // extern "C"
