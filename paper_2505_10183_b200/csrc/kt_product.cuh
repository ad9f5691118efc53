// kt_product.cuh -- matrix products on the tensor cores of sm_100a whose results are worked on before they
// leave the chip: C = A B^T over 16-bit operands with fp32 sums, one tile of C after the other.
//
// Roles of a CTA: one thread brings tiles (TMA) into a ring of shared memory, one issues the matrix instructions,
// and two groups of four warps take the finished sums out of tensor memory, each half of the columns, while the
// next tile is being multiplied into the other of two buffers.  With PAIR two CTAs of a cluster share a tile of 256 x 256: each brings its own
// 128 rows of A and of B and keeps the sums of its own 128 rows of C, and one instruction multiplies in both.  A
// CTA then reads 32 KB for 2 x 128 x 128 x 64 products, half of what it reads alone.  Without it a CTA works on
// 128 x 128 by itself: for products too small to give every pair a tile.
//
// Bound by the tensor cores where the reduction is long: with 2048 elements of it and 12000 tiles they are at work 97 % of the cycles
// (1600 TFLOP/s; a large library product 1670 here), 86 % with 1024 and P to be written.  Small products are bound by
// what a tile costs besides: from the launch before to the first stage 1.1 us, to the last instruction 0.14 us a stage (0.38 for a
// pair's), to the end 2 us (5), to the next launch 0.9; and one CTA alone by the L2, 32 KB a stage at some 64 bytes a cycle.
//
// An operand is a matrix in memory read along its rows (the reduction runs along the row) or down them (the
// reduction runs from row to row).  What lies outside of a matrix arrives as zeros.
//
// A Task says what the tiles are and what becomes of their sums:
//   Params, Maps (descriptions of matrices, nothing else), PAIR, HALF (fp16 operands instead of bf16)
//   Cut(p, worker, workers)      what a worker (a CTA or a pair) does: count() tiles, of which tile(i) is the i-th
//   bool a_down / b_down(tile)   how the operands are read
//   const CUtensorMap *map_a / map_b(maps, cut, tile)
//   int rows_a(cut, tile)        rows that a box of A read along its rows brings: fewer than 128 where the others' results do not matter
//   void finish(p, maps, cut, tile, part)
// Waits are bounded (kt_tensor.cuh).  A tile whose sums never came is finished with NaN in their place.
#pragma once

#include <algorithm>
#include <atomic>
#include <cstring>

#include "kt_internal.h"
#include "kt_tensor.cuh"

namespace {

constexpr int K_STEP = 64;                                // elements of the reduction to a stage: 128 bytes
constexpr int STAGES = 5;
constexpr uint32_t OPERAND_BYTES = TILE * K_STEP * 2, STORE_BYTES = 32 * 128;
constexpr int PRODUCT_THREADS = 384, PRODUCT_LOAD = 0, PRODUCT_ISSUE = 1, PRODUCT_MEMORY = 2, PRODUCT_FINISH = 4;      // warps
constexpr int PRODUCT_SMS = 148;                          // of a B200, one CTA to each

struct Tile {
    int m, n, z, k, steps;                                // first row and column, matrix of the batch, first element and stages of the reduction (0: zeros)
    int kind, share;                                      // the Task's own
};

struct ProductSmem {
    alignas(1024) uint8_t a[STAGES][OPERAND_BYTES], b[STAGES][OPERAND_BYTES], store[8][2][STORE_BYTES];
    uint64_t full[STAGES], free[STAGES], sums_full[2], sums_taken[2];
    uint32_t tmem;
    Patience waits;
};

// ----------------------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t rank_in_pair() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
template <bool PAIR>
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap *map, uint32_t bar, int x, int y, int z) {
    if constexpr (PAIR)       // counted at the barrier of the pair's first CTA
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(to),
                     "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(to),
                     "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, uint32_t from, int x, int y, int z, bool add) {
    if (add)
        asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(from), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(from), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void stores_sent() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }      // the places of those before may be filled again
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

template <bool PAIR>
__device__ __forceinline__ void sums_alloc(uint32_t *to, uint32_t columns) {      // one whole warp (of each CTA)
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tmem_alloc(to, columns);
    }
}
template <bool PAIR>
__device__ __forceinline__ void sums_free(uint32_t at, uint32_t columns) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
    else tmem_free(at, columns);
}
template <bool PAIR>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t word, uint32_t add) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(word), "r"(add) : "memory");
    else
        mma_smem(d, a, b, word, add);
}
// An arrival, in both CTAs of a pair, once every matrix instruction that this thread has issued is done.
template <bool PAIR>
__device__ __forceinline__ void multiplied(uint64_t *bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
    else
        mma_commit(bar);
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {       // a barrier of the cluster
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Words of the matrix instruction and of the operands.  Both operands' rows (or, read down, their 16 K rows) are 128
// bytes in the 128-byte swizzle; read down, chunks of 64 columns are 64 rows apart.
template <bool PAIR, bool HALF>
__device__ __forceinline__ uint32_t product_word(bool a_down, bool b_down) {
    return (1u << 4) | (HALF ? 0u : (1u << 7) | (1u << 10)) | (a_down ? 1u << 15 : 0u) | (b_down ? 1u << 16 : 0u) | (static_cast<uint32_t>((PAIR ? 256 : 128) / 8) << 17) |
           (static_cast<uint32_t>((PAIR ? 256 : 128) / 16) << 24);
}
constexpr uint64_t PRODUCT_DOWN = (static_cast<uint64_t>((K_STEP * 128) >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);

// One operand's part of a stage: 128 rows of 64 elements of the reduction, or 64 rows (of the reduction) of 128.
template <bool PAIR>
__device__ __forceinline__ void load_operand(uint32_t to, const CUtensorMap *map, uint32_t bar, bool down, int row, int k, int z) {
    if (down) {
        load_box<PAIR>(to, map, bar, row, k, z);
        load_box<PAIR>(to + OPERAND_BYTES / 2, map, bar, row + 64, k, z);
    } else {
        load_box<PAIR>(to, map, bar, k, row, z);
    }
}

// ----------------------------------------------------------------------------- finishing
// What a thread of the finishing warps has of a tile: half of a row, and its sums 32 columns at a time.
struct Part {
    int row, col, half;                         // of C: the row, the first column, which half
    uint32_t at;                                // its sums in tensor memory
    uint8_t *store;                             // of the warp: 32 rows of 128 bytes, of two places the one in turn
    int turn;
    int warp_row;                               // the warp's first row of C
    bool there;                                 // else NaN
    bool zero;                                  // nothing to sum
    uint64_t *full;                             // what the sums are waited for with
    uint32_t parity;
    volatile Patience *waits;
    bool waited;
    // The sums are there (a Task may do something else before; over_columns waits by itself).
    __device__ __forceinline__ void wait() {
        if (waited) return;
        waited = true;
        there = there && bar_wait(full, parity, waits);
        tmem_fence_after();
    }
    __device__ __forceinline__ void ask(int c, uint32_t (&r)[32]) const {
        if (there && !zero) tmem_load32(at + c, r);
    }
    __device__ __forceinline__ void get(uint32_t (&r)[32]) const {
        if (there && !zero) {
            tmem_wait_loads(r);
            return;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = there ? 0u : 0x7FFFFFFFu;
    }
    // The 16-byte piece `unit` (0 ... 7) of the thread's row in the store, where the copy engine looks for it.
    __device__ __forceinline__ uint4 *piece(int unit) const {
        const int r = threadIdx.x % 32;
        return reinterpret_cast<uint4 *>(store + r * 128 + ((unit ^ (r & 7)) << 4));
    }
    // The other place, once what was sent from it has been read.
    __device__ __forceinline__ void store_next() {
        if (threadIdx.x % 32 == 0) stores_read_but_one();
        __syncwarp();
        turn ^= 1;
        store += turn ? static_cast<int>(STORE_BYTES) : -static_cast<int>(STORE_BYTES);
    }
    // What the warp has put there goes to (x, y, z); and, from `second` on, to (x2, y2, z) of a second matrix.
    __device__ __forceinline__ void send(const CUtensorMap *map, int x, int y, int z, bool add = false, const CUtensorMap *map2 = nullptr, int second = 0, int x2 = 0, int y2 = 0) const {
        fence_async_smem();
        __syncwarp();
        if (threadIdx.x % 32 == 0) {
            store_box(map, smem_addr(store), x, y, z, add);
            if (map2 != nullptr) store_box(map2, smem_addr(store) + second, x2, y2, z, false);
            stores_sent();
        }
    }
};

// f(column of C, whether it is the second of two, sums of 32 columns) for COLS columns of the thread's row, 64 at a time; the
// next columns are on their way meanwhile.
template <int N>
struct Constant {
    __device__ constexpr operator int() const { return N; }
};
template <int COLS, typename F>
__device__ __forceinline__ void over_columns(Part &part, F f) {
    uint32_t r[2][32];
    part.wait();
    __syncwarp();
    part.ask(0, r[0]);
#pragma unroll 1
    for (int c = 0; c < COLS; c += 64) {
        part.get(r[0]);
        part.ask(c + 32, r[1]);
        f(part.col + c, Constant<0>(), r[0]);
        __syncwarp();           // tensor memory is read by whole warps
        part.get(r[1]);
        if (c + 64 < COLS) part.ask(c + 64, r[0]);
        f(part.col + c + 32, Constant<1>(), r[1]);
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------------- kernel
template <class Task>
__global__ void __launch_bounds__(PRODUCT_THREADS, 1) k_product(const __grid_constant__ typename Task::Maps maps, const __grid_constant__ typename Task::Params p, const uint64_t wait_ns) {
    constexpr bool PAIR = Task::PAIR;
    constexpr int SIDE = PAIR ? 256 : 128;
    constexpr uint32_t COLUMNS = 2 * SIDE;                // of tensor memory: two tiles
    extern __shared__ uint8_t raw[];
    auto &sm = *reinterpret_cast<ProductSmem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = PAIR ? rank_in_pair() : 0;
    const int worker = PAIR ? blockIdx.x / 2 : blockIdx.x, workers = PAIR ? gridDim.x / 2 : gridDim.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) bar_init(&sm.full[i], 1), bar_init(&sm.free[i], 1);
        for (int i = 0; i < 2; ++i) bar_init(&sm.sums_full[i], 1), bar_init(&sm.sums_taken[i], PAIR ? 16 : 8);
        sm.waits = {wait_ns, 0};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == PRODUCT_LOAD && lane < static_cast<int>(sizeof(maps) / sizeof(CUtensorMap)))
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(reinterpret_cast<const CUtensorMap *>(&maps) + lane)) : "memory");
    if (warp == PRODUCT_MEMORY) sums_alloc<PAIR>(&sm.tmem, COLUMNS);
    tmem_fence_before();
    if constexpr (PAIR) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = sm.tmem;
    volatile Patience *waits = &sm.waits;
    after_previous();
    let_next_begin();           // (not before: a chain of small products would come up all at once and wait on every SM)
    const typename Task::Cut cut(p, worker, workers);
    const int tiles = cut.count();

    if (warp == PRODUCT_LOAD) {
        if (lane == 0) {
            uint32_t stage = 0, round = 0;
            bool ok = true;
            for (int i = 0; ok && i < tiles; ++i) {
                const Tile t = cut.tile(i);
                const CUtensorMap *const map_a = Task::map_a(maps, cut, t), *const map_b = Task::map_b(maps, cut, t);
                const int m = t.m + static_cast<int>(rank) * TILE, n = t.n + static_cast<int>(rank) * TILE;
                const uint32_t bytes = (Task::a_down(t) ? OPERAND_BYTES : Task::rows_a(cut, t) * (K_STEP * 2)) + OPERAND_BYTES;
                for (int s = 0; s < t.steps; ++s) {
                    if (!(ok = bar_wait_one(&sm.free[stage], (round + 1) & 1, waits))) break;
                    const uint32_t bar = PAIR ? address_in(smem_addr(&sm.full[stage]), 0) : smem_addr(&sm.full[stage]);
                    if (rank == 0) bar_expect(&sm.full[stage], PAIR ? 2 * bytes : bytes);
                    const int k = t.k + s * K_STEP;
                    load_operand<PAIR>(smem_addr(sm.a[stage]), map_a, bar, Task::a_down(t), m, k, t.z);
                    load_operand<PAIR>(smem_addr(sm.b[stage]), map_b, bar, Task::b_down(t), n, k, t.z);
                    if (++stage == STAGES) stage = 0, ++round;
                }
            }
        }
    } else if (warp == PRODUCT_ISSUE) {
        if (rank == 0 && elected()) {
            uint32_t stage = 0, round = 0;
            bool ok = true;
            for (int i = 0; ok && i < tiles; ++i) {
                const Tile t = cut.tile(i);
                const bool a_down = Task::a_down(t), b_down = Task::b_down(t);
                const uint32_t word = product_word<PAIR, Task::HALF>(a_down, b_down), step_a = a_down ? 2048 >> 4 : 32 >> 4, step_b = b_down ? 2048 >> 4 : 32 >> 4;
                const uint64_t word_a = a_down ? PRODUCT_DOWN : OPERAND_ALONG, word_b = b_down ? PRODUCT_DOWN : OPERAND_ALONG;
                if (!(ok = bar_wait_one(&sm.sums_taken[i & 1], (i / 2 + 1) & 1, waits))) break;
                tmem_fence_after();
                const uint32_t d = tmem + (i & 1) * SIDE;
                for (int s = 0; s < t.steps; ++s) {
                    if (!(ok = bar_wait_one(&sm.full[stage], round & 1, waits))) break;
                    tmem_fence_after();
                    const uint64_t a = operand(word_a, smem_addr(sm.a[stage]));
                    const uint64_t b = operand(word_b, smem_addr(sm.b[stage]));
#pragma unroll
                    for (uint32_t k = 0; k < K_STEP / 16; ++k) multiply<PAIR>(d, a + k * step_a, b + k * step_b, word, s > 0 || k > 0);
                    multiplied<PAIR>(&sm.free[stage]);
                    if (++stage == STAGES) stage = 0, ++round;
                }
                if (ok) multiplied<PAIR>(&sm.sums_full[i & 1]);
            }
        }
    } else if (warp >= PRODUCT_FINISH) {
        const uint32_t group = (warp - PRODUCT_FINISH) / 4, quarter = warp % 4;
        Part part;
        part.half = static_cast<int>(group);
        part.store = sm.store[warp - PRODUCT_FINISH][0], part.turn = 0;
        part.there = true, part.waits = waits;
        for (int i = 0; i < tiles; ++i) {
            const Tile t = cut.tile(i);
            part.warp_row = t.m + static_cast<int>(rank * TILE + quarter * 32);
            part.row = part.warp_row + lane;
            part.zero = t.steps == 0;
            part.col = t.n + static_cast<int>(group) * (SIDE / 2);
            part.at = tmem + (i & 1) * SIDE + group * (SIDE / 2) + ((quarter * 32) << 16);
            part.full = &sm.sums_full[i & 1], part.parity = i / 2 & 1, part.waited = false;
            Task::finish(p, maps, cut, t, part);
            part.wait();
            if (part.there) {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(PAIR ? address_in(smem_addr(&sm.sums_taken[i & 1]), 0) : smem_addr(&sm.sums_taken[i & 1]));
            }
        }
        if (lane == 0) stores_done();
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (waits->gave_up) {       // copies and products in flight get two milliseconds to finish before the memory that they write is handed back
        const uint64_t start = now_ns();
        for (int i = 0; i < 100000 && now_ns() - start < 2000000; ++i) __nanosleep(1000);
    }
    if constexpr (PAIR) cluster_sync();         // the other CTA's copies, products and arrivals that end here are done
    tmem_fence_after();
    if (warp == PRODUCT_MEMORY) sums_free<PAIR>(tmem, COLUMNS);
}

// ---------------------------------------------------------------------------------- host side
// Matrix z of [matrices][rows][cols], pitches in bytes; boxes of box_cols x box_rows whose rows of 128 (64) bytes are in the
// 128-byte (64-byte) swizzle, or as they are.
inline int describe_matrix(CUtensorMap *map, const char *what, CUtensorMapDataType type, int size, const void *at, int64_t cols, int64_t rows, int64_t matrices, int64_t pitch,
                           int64_t matrix_pitch, int box_cols, int box_rows, bool swizzled = true) {
    const encode_fn encode = encoder();
    if (encode == nullptr) return ktd::fail(KT_ERR_CUDA, "the driver does not offer cuTensorMapEncodeTiled");
    const cuuint64_t sizes[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(matrices)};
    const cuuint64_t strides[2] = {rows > 1 ? static_cast<cuuint64_t>(pitch) : 16, matrices > 1 ? static_cast<cuuint64_t>(matrix_pitch) : 16};      // that of a dimension of one is never used
    const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 1}, step[3] = {1, 1, 1};
    const CUtensorMapSwizzle swizzle = !swizzled ? CU_TENSOR_MAP_SWIZZLE_NONE : box_cols * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    const CUresult rc = encode(map, type, 3, const_cast<void *>(at), sizes, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc != CUDA_SUCCESS) return ktd::fail(KT_ERR_CUDA, "describing %s to the copy engine failed with driver status %d", what, static_cast<int>(rc));
    return KT_OK;
}
// An operand of 16-bit elements, read along its rows (box_rows at a time) or down them.
inline int describe_operand(CUtensorMap *map, const char *what, bool half, bool down, const void *at, int64_t cols, int64_t rows, int64_t matrices, int64_t pitch, int64_t matrix_pitch, int box_rows = TILE) {
    return describe_matrix(map, what, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, at, cols, rows, matrices, pitch, matrix_pitch, 64, down ? K_STEP : box_rows);
}

// Starts a product of at most `tiles` tiles: behind a kernel of the same call, or as the call's first, which may not begin
// before all that is in the stream has ended.
template <class Task>
int start_product(typename Task::Maps maps, const typename Task::Params &p, int64_t tiles, cudaStream_t st, bool behind = true) {
    static std::atomic<uint64_t> raised{0};      // a bit for each device on which the kernel's limit has been raised
    constexpr size_t bytes = sizeof(ProductSmem) + 1024;
    static_assert(bytes <= 227 * 1024, "the ring and the stores have to fit");
    int dev = 0;
    KT_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
        KT_CUDA(cudaFuncSetAttribute(k_product<Task>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
        raised.fetch_or(bit, std::memory_order_relaxed);
    }
    if (tiles == 0) return KT_OK;
    // every description is fetched ahead, so those that the Task does not use are copies of one that it does
    const CUtensorMap none{};
    CUtensorMap *const first = reinterpret_cast<CUtensorMap *>(&maps), *const past = first + sizeof(maps) / sizeof(CUtensorMap);
    const CUtensorMap *described = std::find_if(first, past, [&](const CUtensorMap &m) { return std::memcmp(&m, &none, sizeof(m)) != 0; });
    if (described == past) return ktd::fail(KT_ERR_INVALID, "a product without operands");
    for (CUtensorMap *m = first; m < past; ++m)
        if (std::memcmp(m, &none, sizeof(none)) == 0) *m = *described;
    constexpr int CTAS = Task::PAIR ? 2 : 1;
    const int64_t places = PRODUCT_SMS / CTAS;
    const dim3 grid(static_cast<unsigned>(CTAS * (tiles < places ? tiles : places)));
    if (behind) KT_CUDA(launch_behind(k_product<Task>, CTAS, grid, dim3(PRODUCT_THREADS), bytes, st, maps, p, ktd::wait_limit_ns()));
    else KT_CUDA(launch_joint(k_product<Task>, CTAS, grid, dim3(PRODUCT_THREADS), bytes, st, maps, p, ktd::wait_limit_ns()));
    return KT_OK;
}

}  // namespace
