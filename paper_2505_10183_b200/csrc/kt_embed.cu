// kt_embed.cu -- rows of a table for the tokens of a batch, and the table's gradient.  Contracts: include/kaitian.h.
//
//   forward    out_i = scale w[ids_i]
//   backward   dw_v = [base_v +] scale sum over the tokens i with ids_i = v of dout_i
// Both are bound by memory.  The gradient is summed from a list of the tokens in which those of one row stand next to
// each other, in their order in the batch; the list is cut into pieces of equal length whatever the text, and a row
// whose tokens fall into several pieces is joined from their sums.  No atomics on data: the same inputs give the same bits.
#include "../../include/kaitian.h"

#include <cuda_bf16.h>

#include <algorithm>

#include "kt_eight.cuh"
#include "kt_internal.h"

using namespace ktd;

namespace {

constexpr int SMS = 148;                        // of a B200
constexpr int64_t MAX_TOKENS = INT64_C(1) << 30, MAX_VOCAB = 1 << 24, MAX_COLS = 1 << 24;

// Places of a row: its columns, in eights, or (spread) in blocks of 256.
template <bool WHOLE>
__host__ __device__ inline int64_t places_of(int64_t cols) { return WHOLE ? (cols + 7) / 8 * 8 : (cols + 255) / 256 * 256; }

__device__ __forceinline__ void zeros(float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
}

// ------------------------------------------------------------------------------------ forward
struct LookupParams {
    const int64_t *ids;
    const void *weight;
    void *out;
    int64_t weight_stride, out_stride, tokens, cols;
    int vocab;
    float scale;
};

// A warp takes 1024 columns of a token, four pieces to a lane that are asked for before the first is used.  Bound by memory: 16384 tokens
// of 4096 bf16 in 44 us, 6.1 TB/s, 0.93 of a copy.
template <typename W, typename O, bool WHOLE>
__global__ void __launch_bounds__(256) k_embed_forward(const LookupParams p) {
    const int64_t token = static_cast<int64_t>(blockIdx.x) * 8 + threadIdx.x / 32;
    if (token >= p.tokens) return;
    const int64_t id = p.ids[token], c0 = static_cast<int64_t>(blockIdx.y) * 1024 + threadIdx.x % 32 * 8;
    O *const to = static_cast<O *>(p.out) + token * p.out_stride;
    const bool known = id >= 0 && id < p.vocab;
    const W *const row = static_cast<const W *>(p.weight) + (known ? id : 0) * p.weight_stride;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (known && c0 + i * 256 < places_of<WHOLE>(p.cols)) {
            read_eight<W, WHOLE, !WHOLE>(row, c0 + i * 256, p.cols, v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = id < 0 ? 0.0f : __int_as_float(0x7FFFFFFF);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (c0 + i * 256 >= places_of<WHOLE>(p.cols)) break;
        if (known)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= p.scale;
        write_eight<O, WHOLE, !WHOLE>(to, c0 + i * 256, p.cols, v[i]);
    }
}

// ----------------------------------------------------------------------------------- the list
struct ListParams {
    const int64_t *ids;
    int *token, *row, *count;                   // the list, and its length
    int *past;                                  // where a row's tokens end in the list (0: it has none)
    int n, vocab, owners, most, room;           // owners: CTAs; most: rows of the table to each; room: finds that a warp remembers
    unsigned per;                               // floor(2^32 / owners)
};
constexpr int LIST_THREADS = 512, LIST_WARPS = 16, REMEMBERED = 512, MOST_ROWS = 2048;

// The ids of a CTA are those with the same remainder by the number of CTAs: common tokens, which often lie next to each
// other in a table, are spread.  Every CTA goes over all ids: those with a smaller remainder say where its tokens
// begin in the list, so no CTA waits for another.  Counts are kept by row and warp; a warp has the ids of a run of the
// batch, which keeps the order, and remembers those that it found.  Bound by the instructions to an id, and in the CTA of a token that is
// everywhere by those to a find: 16384 ids of which one in eleven is the same token 10 us, 65536 29 (with 96 remembered, 55).
// This CTA's tokens, each handed to put(place, token, id), the places of a row one after the other in the order of the batch; a
// row's first place and tokens to row_is(row of the CTA, place, tokens).  counts: [LIST_WARPS][most], and behind them what is remembered,
// [LIST_WARPS][room] of token and id.  Returns the place past the last.
template <typename RowIs, typename Put>
__device__ __forceinline__ int make_list(const ListParams &p, int *counts, int *sums, bool whole_list, RowIs row_is, Put put) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, mine = blockIdx.x, owners = p.owners;
    for (int i = tid; i < LIST_WARPS * p.most; i += LIST_THREADS) counts[i] = 0;
    __syncthreads();
    int *const of_warp = counts + warp * p.most;
    int2 *const remembered = reinterpret_cast<int2 *>(counts + (LIST_WARPS * p.most + 1) / 2 * 2) + warp * p.room;
    const int run = ((p.n + LIST_WARPS - 1) / LIST_WARPS + 31) / 32 * 32, begin = min(p.n, warp * run), end = min(p.n, begin + run);
    // id -> (row among the CTA's, or -1); smaller: its remainder comes before the CTA's
    auto look = [&](int64_t id, bool &smaller) {
        smaller = false;
        if (id < 0 || id >= p.vocab) return -1;
        unsigned q = __umulhi(static_cast<unsigned>(id), p.per), r = static_cast<unsigned>(id) - q * owners;
        if (r >= static_cast<unsigned>(owners)) ++q, r -= owners;
        smaller = r < static_cast<unsigned>(mine);
        return r == static_cast<unsigned>(mine) ? static_cast<int>(q) : -1;
    };
    int before = 0, found = 0;
    constexpr int TURN = 8;
    int64_t next[TURN];                         // the ids of the turn to come are on their way during this one
    auto ask = [&](int i) {
#pragma unroll
        for (int u = 0; u < TURN; ++u) next[u] = i + u * 32 + lane < end ? p.ids[i + u * 32 + lane] : -1;
    };
    ask(begin);
    for (int i = begin; i < end; i += TURN * 32) {
        int64_t id[TURN];
#pragma unroll
        for (int u = 0; u < TURN; ++u) id[u] = next[u];
        ask(i + TURN * 32);
#pragma unroll
        for (int u = 0; u < TURN; ++u) {
            bool smaller;
            const int q = look(id[u], smaller);
            before += smaller;
            const unsigned mask = __ballot_sync(0xFFFFFFFFu, q >= 0);
            if (mask == 0) continue;            // four times of five, with 148 CTAs
            if (q >= 0) {
                atomicAdd(&of_warp[q], 1);
                const int at = found + __popc(mask & ((1u << lane) - 1));
                if (at < p.room) remembered[at] = make_int2(i + u * 32 + lane, static_cast<int>(id[u]));
            }
            found += __popc(mask);
        }
    }
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    if (lane == 0) sums[warp] = before;
    __syncthreads();
    int base = 0;
    if (whole_list)
        for (int w = 0; w < LIST_WARPS; ++w) base += sums[w];
    __syncthreads();
    // where the tokens of each row and warp begin
    for (int q0 = 0; q0 < p.most; q0 += LIST_THREADS) {
        const int q = q0 + tid;
        int total = 0;
        if (q < p.most)
            for (int w = 0; w < LIST_WARPS; ++w) total += counts[w * p.most + q];
        int up = total;
#pragma unroll
        for (int far = 1; far < 32; far *= 2) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, up, far);
            if (lane >= far) up += x;
        }
        if (lane == 31) sums[warp] = up;
        __syncthreads();
        int at = base + up - total, all = 0;
        for (int w = 0; w < LIST_WARPS; ++w) {
            if (w < warp) at += sums[w];
            all += sums[w];
        }
        base += all;
        if (q < p.most) {
            row_is(q, at, total);
            for (int w = 0; w < LIST_WARPS; ++w) {
                const int here = counts[w * p.most + q];
                counts[w * p.most + q] = at;
                at += here;
            }
        }
        __syncthreads();
    }
    // the tokens to their places, 32 at a time in order: those that were remembered, or the whole run again
    auto place = [&](int token, int64_t id) {
        bool smaller;
        const int q = look(id, smaller);
        if (__ballot_sync(0xFFFFFFFFu, q >= 0) == 0) return;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, q);
        const int rank = __popc(same & ((1u << lane) - 1));
        if (q >= 0) put(of_warp[q] + rank, token, static_cast<int>(id));
        __syncwarp();
        if (q >= 0 && rank == 0) of_warp[q] += __popc(same);
        __syncwarp();
    };
    if (found <= p.room) {
        for (int i = 0; i < found; i += 32) {
            const int2 known = i + lane < found ? remembered[i + lane] : make_int2(0, -1);
            place(known.x, known.y);
        }
    } else {
        ask(begin);
        for (int i = begin; i < end; i += TURN * 32) {
            int64_t id[TURN];
#pragma unroll
            for (int u = 0; u < TURN; ++u) id[u] = next[u];
            ask(i + TURN * 32);
#pragma unroll
            for (int u = 0; u < TURN; ++u) place(i + u * 32 + lane, id[u]);
        }
    }
    return base;
}

__global__ void __launch_bounds__(LIST_THREADS) k_embed_list(const ListParams p) {
    extern __shared__ int counts[];
    __shared__ int sums[LIST_WARPS];
    let_next_begin();
    const int past = make_list(
        p, counts, sums, true,
        [&](int q, int at, int total) {
            const int64_t v = static_cast<int64_t>(q) * p.owners + blockIdx.x;
            if (v < p.vocab) p.past[v] = total > 0 ? at + total : 0;
        },
        [&](int at, int token, int id) { p.token[at] = token, p.row[at] = id; });
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *p.count = past;
}

// ------------------------------------------------------------------------------------ the sums
struct SumParams {
    const int *token, *row, *count;
    const int *past;
    const void *dout, *base;
    void *dweight;
    float *parts;                               // [pieces][2][pitch]: of the row that began before, and of the one that goes on
    int64_t dout_stride, base_stride, dweight_stride, cols, pitch;
    int tokens, length, pieces, across, across_join;    // all tokens, those of a piece, pieces, CTAs across a row
    int vocab, rows_each;                       // rows of the table to a CTA that fills
    float scale;
};
constexpr int MAX_LENGTH = 256, AHEAD = 4;

// Rows of the table that no token has: zeros, or the base's; a row to a warp at a time.
template <typename T, bool WHOLE>
__device__ __forceinline__ void fill_rows(const SumParams &p, int64_t first) {
    const int rows = static_cast<int>(min(static_cast<int64_t>(p.rows_each), p.vocab - first)), lane = threadIdx.x % 32, warps = blockDim.x / 32, vectors = static_cast<int>(places_of<WHOLE>(p.cols) / 8);
    const unsigned empty = __ballot_sync(0xFFFFFFFFu, lane < rows && p.past[first + min(lane, rows - 1)] == 0);
    int nth = -1;
    for (unsigned left = empty; left != 0; left &= left - 1) {
        if (++nth % warps != static_cast<int>(threadIdx.x) / 32) continue;
        const int64_t row = first + __ffs(static_cast<int>(left)) - 1;
        T *const to = static_cast<T *>(p.dweight) + row * p.dweight_stride;
        const T *const like = p.base != nullptr ? static_cast<const T *>(p.base) + row * p.base_stride : nullptr;
        for (int c0 = lane; c0 < vectors; c0 += 4 * 32) {
            Raw<T, WHOLE, !WHOLE> v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                v[u] = {};
                if (like != nullptr && c0 + u * 32 < vectors) v[u].read(like, (c0 + u * 32) * static_cast<int64_t>(8), p.cols);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c0 + u * 32 < vectors) {
                    float x[8];
                    zeros(x);
                    v[u].add_to(x);
                    write_eight<T, WHOLE, !WHOLE>(to, (c0 + u * 32) * static_cast<int64_t>(8), p.cols, x);
                }
        }
    }
}

// A piece of the list to a CTA, eight columns to a thread, AHEAD rows of dout (and of the base, where a row's tokens
// end) on their way at a time.  (16384 tokens of 2048 bf16: 27 us for 120 MB read and written, latency of its rounds; in pieces for two
// rounds of CTAs 30.)
template <typename D, typename T, bool WHOLE>
__global__ void __launch_bounds__(256, 3) k_embed_sum(const SumParams p) {
    __shared__ int token[MAX_LENGTH], row[MAX_LENGTH + 2];       // row[0], row[n + 1]: the neighbours' (-1: none)
    let_next_begin();
    after_previous();
    const int piece = blockIdx.x / p.across, begin = piece * p.length;
    const int all = *p.count, n = min(p.length, all - begin);
    for (int i = threadIdx.x; i < p.length + 2; i += blockDim.x) {       // (asked for at once; what lies past the list's end is not used)
        const int at = begin + i - 1;
        const bool inside = at >= 0 && at < p.tokens;
        const int r = inside ? p.row[at] : -1, t = inside ? p.token[at] : 0;
        row[i] = at < all ? r : -1;
        if (i >= 1 && i <= p.length) token[i - 1] = t;
    }
    if (n <= 0) return;
    __syncthreads();
    const int64_t c = (static_cast<int64_t>(blockIdx.x - piece * p.across) * blockDim.x + threadIdx.x) * 8;
    if (c >= places_of<WHOLE>(p.cols)) return;
    const D *const dout = static_cast<const D *>(p.dout);
    const T *const base = static_cast<const T *>(p.base);
    float sum[8];
    zeros(sum);
    bool whole = row[0] != row[1];              // the row's tokens begin in this piece
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        Raw<D, WHOLE, !WHOLE> v[AHEAD];
        Raw<T, WHOLE, !WHOLE> before[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u;
            if (i < n) v[u].read(dout + token[i] * p.dout_stride, c, p.cols);
            before[u] = {};
            if (base != nullptr && i < n && row[i + 2] != row[i + 1]) before[u].read(base + row[i + 1] * p.base_stride, c, p.cols);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u;
            if (i >= n) break;
            v[u].add_to(sum);
            const int now = row[i + 1], next = row[i + 2];
            if (next == now && i + 1 < n) continue;
            if (whole && next != now) {
                float x[8];
                zeros(x);
                before[u].add_to(x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(sum[e], p.scale, x[e]);
                write_eight<T, WHOLE, !WHOLE>(static_cast<T *>(p.dweight) + now * p.dweight_stride, c, p.cols, x);
            } else {
                float *const to = p.parts + (static_cast<int64_t>(piece) * 2 + (whole ? 1 : 0)) * p.pitch + c;       // pitch: whole vectors
                *reinterpret_cast<float4 *>(to) = make_float4(sum[0], sum[1], sum[2], sum[3]);
                *reinterpret_cast<float4 *>(to + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
            }
            zeros(sum);
            whole = true;
        }
    }
}

// A row whose tokens go on behind the piece in which they begin: that piece's sum, then the next ones', in order, four
// columns to a thread and up to JOINED pieces on their way at a time.  Behind the CTAs of the pieces come those that fill the
// rows without tokens: a row of many tokens, which one or two CTAs join, does not hold up the memory.  (50257 rows of 2048 bf16 with
// a base: 61 us, 6.3 TB/s.)
constexpr int JOINED = 16;
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256) k_embed_join(const SumParams p) {
    let_next_begin();
    after_previous();
    const int joining = p.pieces > 1 ? p.pieces * p.across_join : 0;
    if (static_cast<int>(blockIdx.x) >= joining) {
        fill_rows<T, WHOLE>(p, (static_cast<int64_t>(blockIdx.x) - joining) * p.rows_each);
        return;
    }
    const int mine = blockIdx.x / p.across_join, begin = mine * p.length, end = begin + p.length, all = *p.count;
    if (end >= p.tokens) return;
    const int row = p.row[end - 1], next = p.row[end], before = begin > 0 ? p.row[begin - 1] : -1;       // (asked for at once)
    if (end >= all || next != row || before == row) return;
    const int64_t c = (static_cast<int64_t>(blockIdx.x - mine * p.across_join) * blockDim.x + threadIdx.x) * 4;
    if (c >= places_of<WHOLE>(p.cols)) return;
    const float *const parts = p.parts + c;
    const int64_t last = (p.past[row] - 1) / p.length;       // the piece in which the row's tokens end
    float4 sum = *reinterpret_cast<const float4 *>(parts + (static_cast<int64_t>(mine) * 2 + 1) * p.pitch);
    for (int64_t piece = mine + 1; piece <= last; piece += JOINED) {
        float4 v[JOINED];
#pragma unroll
        for (int u = 0; u < JOINED; ++u)       // (past the last: that again, and not added)
            v[u] = *reinterpret_cast<const float4 *>(parts + min(piece + u, last) * 2 * p.pitch);
#pragma unroll
        for (int u = 0; u < JOINED; ++u)
            if (piece + u <= last) sum.x += v[u].x, sum.y += v[u].y, sum.z += v[u].z, sum.w += v[u].w;
    }
    const float add[4] = {sum.x, sum.y, sum.z, sum.w};
    T *const to = static_cast<T *>(p.dweight) + row * p.dweight_stride;
    const T *const base = p.base != nullptr ? static_cast<const T *>(p.base) + row * p.base_stride : nullptr;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t at = column_of<!WHOLE>(c & ~static_cast<int64_t>(7), static_cast<int>(c & 7) + e);
        if (at < p.cols) {
            const float x = fmaf(add[e], p.scale, base != nullptr ? static_cast<float>(base[at]) : 0.0f);
            if constexpr (sizeof(T) == 2) to[at] = __float2bfloat16_rn(x);
            else to[at] = x;
        }
    }
}

// Few tokens: all in one launch, since three of them take longer than their work.  A CTA makes the list of its own tokens in
// shared memory and then its own rows: a group of warps that spans a row's columns takes a row at a time, and rows of more
// than ALONE tokens are shared by all groups, whose sums are added in order.  (999 tokens, 500 columns, fp32, a table of
// 8001 rows: 16.4 us in three launches, 12.3 so.)
constexpr int DIRECT_TOKENS = 2048, ALONE = 8;
constexpr int64_t DIRECT_ELEMENTS = INT64_C(1) << 20;      // a row that most tokens share is read by one CTA

template <typename D, typename T, bool WHOLE>
__global__ void __launch_bounds__(LIST_THREADS) k_embed_direct(const ListParams l, const SumParams p) {
    extern __shared__ int counts[];             // as make_list has it, then the rows' first places and the end
    __shared__ int list_sums[LIST_WARPS], token[DIRECT_TOKENS];
    __shared__ float4 sums[LIST_THREADS][2];
    __shared__ int shared_rows[DIRECT_TOKENS / ALONE], shared_count;       // rows of more than ALONE tokens, in any order
    if (threadIdx.x == 0) shared_count = 0;
    int *const starts = counts + (LIST_WARPS * l.most + 1) / 2 * 2 + 2 * LIST_WARPS * l.room;
    const int last = make_list(
        l, counts, list_sums, false,
        [&](int q, int at, int n) {
            starts[q] = at;
            if (n > ALONE) shared_rows[atomicAdd(&shared_count, 1)] = q;
        },
        [&](int at, int t, int) { token[at] = t; });
    if (threadIdx.x == 0) starts[l.most] = last;
    __syncthreads();
    const int vectors = static_cast<int>(places_of<WHOLE>(p.cols) / 8), span = min(LIST_THREADS, (vectors + 31) / 32 * 32), groups = LIST_THREADS / span, group = threadIdx.x / span, lane = threadIdx.x - group * span;
    const D *const dout = static_cast<const D *>(p.dout);
    const T *const base = static_cast<const T *>(p.base);
    auto add = [&](int from, int past, int64_t c, float (&sum)[8]) {
        for (int i0 = from; i0 < past; i0 += ALONE) {
            Raw<D, WHOLE, !WHOLE> v[ALONE];
#pragma unroll
            for (int u = 0; u < ALONE; ++u)
                if (i0 + u < past) v[u].read(dout + token[i0 + u] * p.dout_stride, c, p.cols);
#pragma unroll
            for (int u = 0; u < ALONE; ++u)
                if (i0 + u < past) v[u].add_to(sum);
        }
    };
    auto write = [&](int64_t row, int64_t c, const float (&sum)[8]) {
        Raw<T, WHOLE, !WHOLE> before = {};
        if (base != nullptr) before.read(base + row * p.base_stride, c, p.cols);
        float x[8];
        zeros(x);
        before.add_to(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(sum[e], p.scale, x[e]);
        write_eight<T, WHOLE, !WHOLE>(static_cast<T *>(p.dweight) + row * p.dweight_stride, c, p.cols, x);
    };
    for (int i = 0; i < shared_count; ++i) {
        const int q = shared_rows[i], from = starts[q], n = starts[q + 1] - from;
        for (int v0 = 0; v0 < vectors; v0 += span) {
            const int64_t c = (v0 + lane) * static_cast<int64_t>(8);
            float sum[8];
            zeros(sum);
            if (group < groups && c < places_of<WHOLE>(p.cols)) add(from + n * group / groups, from + n * (group + 1) / groups, c, sum);
            __syncthreads();
            sums[threadIdx.x][0] = make_float4(sum[0], sum[1], sum[2], sum[3]), sums[threadIdx.x][1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
            __syncthreads();
            if (group > 0 || c >= places_of<WHOLE>(p.cols)) continue;
            for (int g = 1; g < groups; ++g) {
                const float4 a = sums[g * span + lane][0], b = sums[g * span + lane][1];
                sum[0] += a.x, sum[1] += a.y, sum[2] += a.z, sum[3] += a.w, sum[4] += b.x, sum[5] += b.y, sum[6] += b.z, sum[7] += b.w;
            }
            write(static_cast<int64_t>(q) * l.owners + blockIdx.x, c, sum);
        }
    }
    if (group >= groups) return;
    const int rows = min(l.most, (l.vocab - static_cast<int>(blockIdx.x) + l.owners - 1) / l.owners);      // the CTA's
    for (int q = group; q < rows; q += groups) {
        const int from = starts[q], n = starts[q + 1] - from;
        if (n > ALONE || (n == 0 && p.base == p.dweight)) continue;       // (an untouched row of the gradient that is there)
        for (int v = lane; v < vectors; v += span) {
            float sum[8];
            zeros(sum);
            add(from, from + n, v * static_cast<int64_t>(8), sum);
            write(static_cast<int64_t>(q) * l.owners + blockIdx.x, v * static_cast<int64_t>(8), sum);
        }
    }
}

// ---------------------------------------------------------------------------------- host side
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// How the gradient's work is cut: from the sizes alone.
struct Plan {
    int64_t owners, most, room, threads, across, threads_join, across_join, length, pieces, pitch, at_row, at_past, at_parts, bytes;
    Plan(int64_t tokens, int64_t cols, int64_t vocab, bool whole) {
        // a CTA for each SM, more where a CTA's counts would not fit its shared memory
        owners = std::max<int64_t>(SMS, (vocab + MOST_ROWS - 1) / MOST_ROWS), most = (vocab + owners - 1) / owners;
        room = std::min<int64_t>(REMEMBERED, up((tokens + LIST_WARPS - 1) / LIST_WARPS, 32));
        const int64_t places = whole ? places_of<true>(cols) : places_of<false>(cols), vectors = places / 8, fours = places / 4;
        threads = std::min<int64_t>(256, up(vectors, 32)), across = (vectors + threads - 1) / threads;
        threads_join = std::min<int64_t>(256, up(fours, 32)), across_join = (fours + threads_join - 1) / threads_join;
        // one round of three CTAs of 256 threads to an SM (what its registers hold), but short pieces leave more rows to be joined
        length = std::min<int64_t>(MAX_LENGTH, std::max<int64_t>(8, (tokens * across + SMS * 3 * 256 / threads - 1) / (SMS * 3 * 256 / threads)));
        pieces = (tokens + length - 1) / length;
        pitch = places;
        int64_t at = 1024 + up(tokens * 4, 1024);      // the list's length and tokens
        at_row = at, at += up(tokens * 4, 1024);
        at_past = at, at += up(vocab * 4, 1024);
        at_parts = at, at += pieces > 1 ? pieces * 2 * pitch * 4 : 0;
        bytes = at;
    }
};

int64_t bytes_needed(int64_t tokens, int64_t cols, int64_t vocab) { return std::max(Plan(tokens, cols, vocab, true).bytes, Plan(tokens, cols, vocab, false).bytes); }

// (Rows that are only read may overlap, or be one row with a stride of 0.)
int check_matrix(const char *what, const void *at, int64_t stride, int64_t rows, int64_t cols, int dtype, bool written) {
    if (rows == 0 || cols == 0) return KT_OK;
    if (at == nullptr) return fail(KT_ERR_INVALID, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(at) % (dtype == KT_F32 ? 4 : 2)) return fail(KT_ERR_ALIGN, "%s is not aligned to its elements", what);
    if (rows > 1 && (stride < (written ? cols : 0) || stride > INT64_C(1) << 38)) return fail(KT_ERR_SHAPE, "%s: rows of %lld elements cannot be %lld apart", what, (long long)cols, (long long)stride);
    return KT_OK;
}
int check_common(int64_t tokens, int64_t cols, int64_t vocab, int dtype, int param_dtype, float scale, const int64_t *ids) {
    for (int t : {dtype, param_dtype})
        if (t != KT_F32 && t != KT_BF16) return fail(KT_ERR_INVALID, "unknown dtype %d", t);
    if (tokens < 0 || tokens > MAX_TOKENS || cols < 1 || cols > MAX_COLS || vocab < 1 || vocab > MAX_VOCAB)
        return fail(KT_ERR_SHAPE, "%lld tokens, %lld columns, a vocabulary of %lld", (long long)tokens, (long long)cols, (long long)vocab);
    if (!(scale - scale == 0.0f)) return fail(KT_ERR_INVALID, "scale must be finite");
    if (tokens > 0 && ids == nullptr) return fail(KT_ERR_INVALID, "ids is NULL");
    if (reinterpret_cast<uintptr_t>(ids) % 8) return fail(KT_ERR_ALIGN, "ids is not aligned to its elements");
    return KT_OK;
}
bool whole(const void *at, int64_t stride, int64_t rows, int dtype) {
    return reinterpret_cast<uintptr_t>(at) % 16 == 0 && (rows <= 1 || stride * (dtype == KT_F32 ? 4 : 2) % 16 == 0);
}

template <typename W, typename O>
int lookup(const LookupParams &p, bool vectors, cudaStream_t st) {
    const dim3 grid(static_cast<unsigned>((p.tokens + 7) / 8), static_cast<unsigned>((p.cols + 1023) / 1024));
    vectors ? k_embed_forward<W, O, true><<<grid, 256, 0, st>>>(p) : k_embed_forward<W, O, false><<<grid, 256, 0, st>>>(p);
    KT_CUDA(cudaGetLastError());
    return KT_OK;
}

template <typename D, typename T, bool WHOLE>
int gradient(const ListParams &l, const SumParams &s, const Plan &plan, cudaStream_t st) {
    const size_t bytes = static_cast<size_t>((LIST_WARPS * plan.most + 1) / 2 * 2 * 4 + LIST_WARPS * l.room * 8);
    constexpr int MOST = LIST_WARPS * (MOST_ROWS * 4 + REMEMBERED * 8);
    if (l.n <= DIRECT_TOKENS && l.n * s.cols <= DIRECT_ELEMENTS) {
        const size_t more = bytes + static_cast<size_t>(plan.most + 1) * 4;
        if (more > 16 * 1024) KT_CUDA(cudaFuncSetAttribute(k_embed_direct<D, T, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, LIST_WARPS * (MOST_ROWS * 4 + DIRECT_TOKENS / LIST_WARPS * 8) + MOST_ROWS * 4 + 4));      // 26 of the 48 KB that need no leave are static
        k_embed_direct<D, T, WHOLE><<<static_cast<unsigned>(plan.owners), LIST_THREADS, more, st>>>(l, s);
        KT_CUDA(cudaGetLastError());
        return KT_OK;
    }
    if (bytes > 40 * 1024) KT_CUDA(cudaFuncSetAttribute(k_embed_list, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST));      // 48 KB need no leave
    k_embed_list<<<static_cast<unsigned>(plan.owners), LIST_THREADS, bytes, st>>>(l);
    KT_CUDA(cudaGetLastError());
    const int64_t summing = plan.pieces * plan.across, fillers = s.base == s.dweight ? 0 : (s.vocab + s.rows_each - 1) / s.rows_each;
    const int64_t ending = (plan.pieces > 1 ? plan.pieces * plan.across_join : 0) + fillers;
    if (summing > INT32_MAX || ending > INT32_MAX) return fail(KT_ERR_SHAPE, "tokens x columns are too many");
    if (summing > 0) KT_CUDA(launch_behind(k_embed_sum<D, T, WHOLE>, 1, dim3(static_cast<unsigned>(summing)), dim3(static_cast<unsigned>(plan.threads)), 0, st, s));
    if (ending > 0) KT_CUDA(launch_behind(k_embed_join<T, WHOLE>, 1, dim3(static_cast<unsigned>(ending)), dim3(static_cast<unsigned>(plan.threads_join)), 0, st, s));
    return KT_OK;
}

}  // namespace

extern "C" {

int kt_embed_forward(const int64_t *ids, const void *weight, int64_t weight_stride, int param_dtype, void *out, int64_t out_stride, int64_t tokens, int64_t cols, int64_t vocab, int dtype, float scale,
                     void *stream) {
    if (int rc = check_common(tokens, cols, vocab, dtype, param_dtype, scale, ids)) return rc;
    if (tokens == 0) return KT_OK;
    if (int rc = check_matrix("weight", weight, weight_stride, vocab, cols, param_dtype, false)) return rc;
    if (int rc = check_matrix("out", out, out_stride, tokens, cols, dtype, true)) return rc;
    const LookupParams p{ids, weight, out, weight_stride, out_stride, tokens, cols, static_cast<int>(vocab), scale};
    const bool vectors = whole(weight, weight_stride, vocab, param_dtype) && whole(out, out_stride, tokens, dtype);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (param_dtype == KT_F32) return dtype == KT_F32 ? lookup<float, float>(p, vectors, st) : lookup<float, __nv_bfloat16>(p, vectors, st);
    return dtype == KT_F32 ? lookup<__nv_bfloat16, float>(p, vectors, st) : lookup<__nv_bfloat16, __nv_bfloat16>(p, vectors, st);
}

int64_t kt_embed_workspace(int64_t tokens, int64_t cols, int64_t vocab) {
    if (tokens < 0 || tokens > MAX_TOKENS || cols < 1 || cols > MAX_COLS || vocab < 1 || vocab > MAX_VOCAB) return 0;
    return bytes_needed(tokens, cols, vocab);
}

int kt_embed_backward(const void *dout, int64_t dout_stride, const int64_t *ids, const void *base, int64_t base_stride, void *dweight, int64_t dweight_stride, int param_dtype, void *workspace,
                      int64_t workspace_bytes, int64_t tokens, int64_t cols, int64_t vocab, int dtype, float scale, void *stream) {
    if (int rc = check_common(tokens, cols, vocab, dtype, param_dtype, scale, ids)) return rc;
    if (int rc = check_matrix("dout", dout, dout_stride, tokens, cols, dtype, false)) return rc;
    if (int rc = check_matrix("dweight", dweight, dweight_stride, vocab, cols, param_dtype, true)) return rc;
    if (base != nullptr)
        if (int rc = check_matrix("base", base, base_stride, vocab, cols, param_dtype, false)) return rc;
    if (base == dweight && vocab > 1 && base_stride != dweight_stride) return fail(KT_ERR_SHAPE, "base is dweight, with another stride");
    const bool vectors = (tokens == 0 || whole(dout, dout_stride, tokens, dtype)) && whole(dweight, dweight_stride, vocab, param_dtype) && (base == nullptr || whole(base, base_stride, vocab, param_dtype));
    const Plan plan(tokens, cols, vocab, vectors);
    const int64_t need = bytes_needed(tokens, cols, vocab);
    if (workspace == nullptr) return fail(KT_ERR_INVALID, "workspace is NULL");
    if (workspace_bytes < need) return fail(KT_ERR_SHAPE, "workspace of %lld bytes: %lld are needed", (long long)workspace_bytes, (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(KT_ERR_ALIGN, "workspace is not 16-byte aligned");
    char *const ws = static_cast<char *>(workspace);
    int *const count = reinterpret_cast<int *>(ws), *const token = reinterpret_cast<int *>(ws + 1024), *const row = reinterpret_cast<int *>(ws + plan.at_row);
    int *const past = reinterpret_cast<int *>(ws + plan.at_past);
    const ListParams l{ids, token, row, count, past, static_cast<int>(tokens), static_cast<int>(vocab), static_cast<int>(plan.owners), static_cast<int>(plan.most), static_cast<int>(plan.room),
                       static_cast<unsigned>((UINT64_C(1) << 32) / static_cast<uint64_t>(plan.owners))};
    // CTAs that fill take 64 KB, but a row to each warp at least, and as many as a warp has lanes at most
    const int64_t rows_each = std::min<int64_t>(32, std::max<int64_t>(plan.threads_join / 32, 65536 / (cols * (param_dtype == KT_F32 ? 4 : 2))));
    const SumParams s{token, row, count, past, dout, base, dweight, reinterpret_cast<float *>(ws + plan.at_parts), dout_stride, base_stride, dweight_stride, cols, plan.pitch, static_cast<int>(tokens), static_cast<int>(plan.length),
                      static_cast<int>(plan.pieces), static_cast<int>(plan.across), static_cast<int>(plan.across_join), static_cast<int>(vocab), static_cast<int>(rows_each), scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (param_dtype == KT_F32) {
        if (dtype == KT_F32) return vectors ? gradient<float, float, true>(l, s, plan, st) : gradient<float, float, false>(l, s, plan, st);
        return vectors ? gradient<__nv_bfloat16, float, true>(l, s, plan, st) : gradient<__nv_bfloat16, float, false>(l, s, plan, st);
    }
    if (dtype == KT_F32) return vectors ? gradient<float, __nv_bfloat16, true>(l, s, plan, st) : gradient<float, __nv_bfloat16, false>(l, s, plan, st);
    return vectors ? gradient<__nv_bfloat16, __nv_bfloat16, true>(l, s, plan, st) : gradient<__nv_bfloat16, __nv_bfloat16, false>(l, s, plan, st);
}

}  // extern "C"
