// kt_tensor.cuh -- what a kernel needs to feed the tensor cores of sm_100a: barriers in shared
// memory with bounded waits, tile copies (TMA), tensor memory and its accesses, and the matrix
// instruction on bf16 operands with fp32 sums.
//
// Tiles in shared memory are rows of 64 bf16 (128 bytes) in the 128-byte swizzle, 128 rows to a chunk
// of 16 KB, chunks side by side for wider rows.  A chunk serves as an operand in both
// directions: with the reduction along the row (K-major) or down the rows (MN-major).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace {

constexpr int TILE = 128;                       // rows of a tile: the M and N of the matrix instruction
constexpr uint32_t CHUNK = TILE * 128;          // bytes of 128 rows of 64 bf16

// Waits that gave up since the library was loaded; the results of a kernel that counts here are not valid.
__device__ unsigned long long g_waits_given_up;

// A CTA's waits: how long one may last, and whether one has given up.
struct Patience {
    uint64_t limit_ns;
    uint32_t gave_up;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---------------------------------------------------------------------------------- barriers
__device__ __forceinline__ void bar_init(uint64_t *bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// One arrival for a warp, after what all its lanes have done before.
__device__ __forceinline__ void bar_arrive_warp(uint64_t *bar) {
    __syncwarp();
    if (threadIdx.x % 32 == 0) bar_arrive(bar);
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
// Whether the phase of that parity has ended: at once, and (bar_try) after a while, unless it ends before.
__device__ __forceinline__ bool bar_test(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ bool bar_try(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// Waits for the phase of that parity to end.  False when it gave up, or when another warp of the CTA did: the
// caller then leaves its loop, and the kernel ends.  Called by one thread, or (bar_wait) by whole warps.
// With a limit of 0 whatever is not there at the first look is given up.
__device__ __forceinline__ bool bar_wait_slow(uint64_t *bar, uint32_t parity, volatile Patience *waits) {
    const uint64_t start = now_ns();
    for (uint32_t n = 0;; ++n) {
        if (n % 16 == 0) {
            if (waits->gave_up) return false;
            if (now_ns() - start >= waits->limit_ns) {
                waits->gave_up = 1;
                atomicAdd(&g_waits_given_up, 1ull);
                return false;
            }
        }
        if (bar_try(bar, parity)) return true;
    }
}
__device__ __forceinline__ bool bar_wait_one(uint64_t *bar, uint32_t parity, volatile Patience *waits) {
    return bar_test(bar, parity) || bar_wait_slow(bar, parity, waits);
}
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, volatile Patience *waits) {
    bool ok = bar_test(bar, parity);
    if (!ok) ok = bar_wait_slow(bar, parity, waits);
    return __all_sync(0xFFFFFFFFu, ok);
}

// A group of four warps gives registers back, or takes them, all four together.  What is taken has to have been
// given back out of the block's own registers at launch.
template <int N>
__device__ __forceinline__ void registers_give() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_take() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// ------------------------------------------------------------------------------- tile copies
// [dim, tokens, heads, batch] -> 128 tokens of 64 elements.
__device__ __forceinline__ void copy_tile(uint32_t to, const CUtensorMap *map, uint64_t *bar, int dim, int token, int head, int batch) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(to),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_addr(bar)), "r"(dim), "r"(token), "r"(head), "r"(batch)
        : "memory");
}
// Plain bytes; both addresses and the size are multiples of 16.
__device__ __forceinline__ void copy_bytes(uint32_t to, const void *from, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes),
                 "r"(smem_addr(bar))
                 : "memory");
}
// What threads have written to shared memory becomes visible to the tensor cores and copies.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ------------------------------------------------------------------------------- work to come
// A CTA that stays: one thread finds out what it does next (up to QUEUE items ahead), every role of the CTA
// reads each answer and says so.
constexpr int QUEUE = 4;
struct Queue {
    alignas(16) uint4 answer[QUEUE];
    uint64_t full[QUEUE], free[QUEUE];
};
__device__ __forceinline__ void queue_init(Queue &q, uint32_t readers) {
    for (int i = 0; i < QUEUE; ++i) bar_init(&q.full[i], 1), bar_init(&q.free[i], readers);
}
// Answers from the launch itself: the next block of the grid that has not been started, whose place the
// CTA takes.  (free[k % QUEUE] has been waited for.)
__device__ __forceinline__ void queue_ask(Queue &q, uint32_t k) {
    bar_expect(&q.full[k % QUEUE], sizeof(uint4));
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_addr(&q.answer[k % QUEUE])),
                 "r"(smem_addr(&q.full[k % QUEUE]))
                 : "memory");
}
// The block of answer k, or -1 where there is none left.
__device__ __forceinline__ int queue_read(const Queue &q, uint32_t k) {
    uint32_t x, given;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\t"
        "mov.u32 %0, 0;\n\t"
        "ld.shared.b128 a, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
        "selp.u32 %1, 1, 0, p;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, _, _, _}, a;\n\t}"
        : "=&r"(x), "=&r"(given)
        : "r"(smem_addr(&q.answer[k % QUEUE]))
        : "memory");
    fence_async_smem();
    return given ? static_cast<int>(x) : -1;
}
// Answers from a counter in device memory, where items have to come in their order.
__device__ __forceinline__ void queue_count(Queue &q, uint32_t k, unsigned *counter, unsigned first, int most) {
    const unsigned block = first + atomicAdd(counter, 1u);
    q.answer[k % QUEUE].x = block < static_cast<unsigned>(most) ? block : 0xFFFFFFFFu;
    bar_arrive(&q.full[k % QUEUE]);
}
// For roles of one thread, and of a whole warp.
template <bool COUNTED>
__device__ __forceinline__ int queue_next_one(Queue &q, uint32_t k, volatile Patience *waits) {
    if (!bar_wait_one(&q.full[k % QUEUE], k / QUEUE & 1, waits)) return -1;
    const int block = COUNTED ? static_cast<int>(q.answer[k % QUEUE].x) : queue_read(q, k);
    bar_arrive(&q.free[k % QUEUE]);
    return block;
}
template <bool COUNTED>
__device__ __forceinline__ int queue_next(Queue &q, uint32_t k, volatile Patience *waits) {
    if (!bar_wait(&q.full[k % QUEUE], k / QUEUE & 1, waits)) return -1;
    const int block = COUNTED ? static_cast<int>(q.answer[k % QUEUE].x) : queue_read(q, k);
    bar_arrive_warp(&q.free[k % QUEUE]);
    return block;
}

// ------------------------------------------------------------------------------ tensor memory
__device__ __forceinline__ void tmem_alloc(uint32_t *to, uint32_t columns) {      // one whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {        // the same warp
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
// 32 columns of the 32 lanes that belong to the warp's place in its group of four.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 :
                 : "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
                   "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
                   "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :
                 : "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// The values are tied to the wait, or the compiler could move what uses them ahead of it.
__device__ __forceinline__ void tmem_loaded(uint32_t (&r)[32]) {
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                      "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]),
                      "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                      "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void tmem_wait_loads(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    tmem_loaded(r);
}
template <int N>
__device__ __forceinline__ void tmem_wait_loads(uint32_t (&r)[N][32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) tmem_loaded(r[i]);
}
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Order between tensor memory accesses and barrier traffic: before an arrival, after a wait.
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// -------------------------------------------------------------------------- matrix instruction
// Instruction word: fp32 sums, bf16 operands, M = 128; bit 16 says that B is MN-major.
__host__ __device__ constexpr uint32_t mma_word(int n, bool b_down) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_down ? 1u << 16 : 0u) | (static_cast<uint32_t>(n / 8) << 17) | (static_cast<uint32_t>(TILE / 16) << 24);
}
// Operand words (without the address): groups of 8 rows are 1024 bytes apart; for an MN-major operand
// chunks of 64 elements along the row are CHUNK apart.
constexpr uint64_t OPERAND_ALONG = (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
constexpr uint64_t OPERAND_DOWN = (static_cast<uint64_t>(CHUNK >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
__device__ __forceinline__ uint32_t in_word(uint32_t addr) { return (addr & 0x3FFFF) >> 4; }      // without the CTA's rank in its cluster
__device__ __forceinline__ uint64_t operand(uint64_t word, uint32_t addr) { return word | in_word(addr); }

// One lane of a warp that is whole.
__device__ __forceinline__ bool elected() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t word, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(word), "r"(add)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t word, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(word), "r"(add)
        : "memory");
}
// An arrival once every matrix instruction that this thread has issued is done.
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// D[128 x N] (+)= A B^T over rows of DH elements: both tiles K-major, N rows of B.
template <int DH, int N>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, bool add = false) {
    const uint64_t wa = operand(OPERAND_ALONG, a), wb = operand(OPERAND_ALONG, b);
#pragma unroll
    for (int k = 0; k < DH / 16; ++k) {
        const uint64_t off = ((k / 4) * CHUNK + (k % 4) * 32) >> 4;
        mma_smem(d, wa + off, wb + off, mma_word(N, false), k > 0 ? 1 : static_cast<uint32_t>(add));
    }
}
// D[128 x DH] (+)= A B over ROWS rows of B: A is bf16 in ROWS / 2 columns of tensor memory, B is read down
// its rows.
template <int DH, int ROWS>
__device__ __forceinline__ void product_down(uint32_t d, uint32_t a, uint32_t b, bool add) {
    const uint64_t wb = operand(OPERAND_DOWN, b);
#pragma unroll
    for (int k = 0; k < ROWS / 16; ++k)
        mma_tmem(d, a + k * 8, wb + ((k * 2048) >> 4), mma_word(DH, true), k > 0 ? 1 : static_cast<uint32_t>(add));
}
// D[128 x N] = A B^T over 16 elements a row, of which only the first 8 differ from zero.  Rows of 16 bytes lie one
// after the other; the second 8 elements of all rows are the zeros at `zeros`, past both.
template <int N>
__device__ __forceinline__ void product_short(uint32_t d, uint32_t a, uint32_t b, uint32_t zeros) {
    auto word = [&](uint32_t at) { return (static_cast<uint64_t>((zeros - at) >> 4) << 16) | (static_cast<uint64_t>(128 >> 4) << 32) | (1ull << 46) | in_word(at); };
    mma_smem(d, word(a), word(b), mma_word(N, false), 0);
}

__device__ __forceinline__ float2 pair_of(const uint32_t (&r)[32], int i) { return make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])); }
__device__ __forceinline__ uint32_t pack_bf16(float2 v) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v.y), "f"(v.x));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---------------------------------------------------------------------------------- host side
typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline encode_fn encoder() {
    static const encode_fn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<encode_fn>(f);
    }();
    return fn;
}

}  // namespace
