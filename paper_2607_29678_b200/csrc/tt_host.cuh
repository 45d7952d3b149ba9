// What the entry points that need no vocabulary (scores of ids, block tables) share: types, error returns, launches, the device's size.
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

typedef uint32_t u32;
typedef uint64_t u64;

#define TT_TRY(x) do { if ((x) != cudaSuccess) { cudaGetLastError(); return TT_ERR_CUDA; } } while (0)

// Is one of the addresses no multiple of `align` (a power of two)?
template <typename... P> static inline bool host_misaligned(size_t align, P... p) { return ((((uintptr_t)p) | ...) & (align - 1)) != 0; }

// SMs of the current device, 0 on an error (asked for at every call: an attribute query costs well under a microsecond, and the
// current device may change between calls).
static inline int host_sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
    return n;
}

// Launches `kernel` in clusters of `cluster` CTAs (1: none) so that it may be placed while the kernel before it on the stream drains; every
// CTA waits inside (cudaGridDependencySynchronize) before it touches memory that kernel may write.
template <typename... KernelParams, typename... Params>
static cudaError_t host_launch(void (*kernel)(KernelParams...), unsigned grid, unsigned block, unsigned cluster, size_t smem, cudaStream_t st, const Params&... p) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return cudaLaunchKernelEx(&cfg, kernel, p...);
}

#if defined(__CUDACC__)
// 16 bytes from device to shared memory, both aligned to 16, on their way until the thread has waited for all but the last N of its groups.
__device__ __forceinline__ void copy_async(void* to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((u32)__cvta_generic_to_shared(to)), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }
// Clusters of CTAs: barrier (release / acquire), and writes to the shared memory of CTA `rank` at the place of this CTA's `p`.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ u32 cluster_map(const void* p, u32 rank) {
    u32 r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((u32)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_put(u32 at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void cluster_put(u32 at, u64 v) { asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(at), "l"(v) : "memory"); }
#endif
