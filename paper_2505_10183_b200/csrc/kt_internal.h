// kt_internal.h -- what the translation units of the library share with each other; not part
// of the ABI (that is include/kaitian.h).
#pragma once

#include <cstdint>
#include <vector>

#include "../../include/kaitian.h"

namespace ktd {

// Stores the message kt_last_error() returns to the calling thread; returns `code`.
int fail(int code, const char *fmt, ...);

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Bucket plan (DDP-style bucketing, Section III): tensors in reverse list order, greedy fill up to cap elements, tensors never
// split, every tensor at a multiple of 8 elements, every bucket at a multiple of 64.
struct BucketPlan {
    std::vector<int64_t> offset;      // [T] list order
    std::vector<int32_t> bucket_of;   // [T] list order
    std::vector<int64_t> start;       // [n_buckets]
    std::vector<int> u_lo, u_hi;      // transport-order tensor range of each bucket
    int64_t total = 0;
};

void plan_buckets(const int64_t *numel, int T, int64_t bucket_cap_bytes, BucketPlan *bp);

// Member m of M owns units [floor(m U / M), floor((m + 1) U / M)) of a range of U work units.
void member_units(int64_t U, int member, int M, int64_t *first, int64_t *past);

// KT_OK, or KT_ERR_INVALID with a message when a share is missing or below one.
int check_shares(const int32_t *shares, int K);

// How long a wait inside a kernel may last (kt_attn_wait_limit), and how many gave up on the current device in the
// kernels of the other files that wait (kt_waits_given_up).
uint64_t wait_limit_ns();
int xent_given_up(unsigned long long *count);
int orth_given_up(unsigned long long *count);

}  // namespace ktd

#ifdef __CUDACC__
template <typename... Params, typename... Args>
cudaError_t launch_with(cudaLaunchAttribute *attrs, int n, void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchConfig_t config{};
    config.gridDim = grid, config.blockDim = block, config.dynamicSmemBytes = smem, config.stream = stream;
    config.attrs = attrs, config.numAttrs = n;
    return cudaLaunchKernelEx(&config, kernel, args...);
}
// A launch whose blocks come in clusters of `joint`, next to each other in x.
template <typename... Params, typename... Args>
cudaError_t launch_joint(void (*kernel)(Params...), unsigned joint, dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute cluster{};
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = joint, cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    return launch_with(&cluster, 1, kernel, grid, block, smem, stream, args...);
}
// A launch that may begin while the one before it in the stream ends: its blocks come up as places become
// free, and call after_previous() before they touch what the one before writes.  In clusters where joint > 1.
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), unsigned joint, dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute attrs[2] = {};
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = joint, attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    return launch_with(attrs, joint > 1 ? 2 : 1, kernel, grid, block, smem, stream, args...);
}
// A barrier of the cluster's threads, and values in another CTA's shared memory, at this one's address.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
}
__device__ __forceinline__ uint32_t address_in(uint32_t mine, unsigned rank) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(rank));
    return at;
}
__device__ __forceinline__ float of_cta(uint32_t mine, unsigned rank) {
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(address_in(mine, rank)) : "memory");
    return x;
}
__device__ __forceinline__ float2 of_cta2(uint32_t mine, unsigned rank) {
    float2 x;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(address_in(mine, rank)) : "memory");
    return x;
}
__device__ __forceinline__ float4 of_cta4(uint32_t mine, unsigned rank) {
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(address_in(mine, rank)) : "memory");
    return x;
}
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
#endif

#define KT_CUDA(call)                                                                       \
    do {                                                                                    \
        cudaError_t e_ = (call);                                                            \
        if (e_ != cudaSuccess)                                                              \
            return ::ktd::fail(KT_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));       \
    } while (0)
