// Clusters of CTAs: barriers, values in another CTA's shared memory, launches.
#pragma once
#include "cache_view.cuh"

namespace amoeba {

constexpr int kMaxCluster = 8;

__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(r));
    return r;
}
// A 32-bit value at the same place in another CTA's shared memory.
__device__ __forceinline__ int32_t load_remote(const int32_t* p, uint32_t rank) {
    uint32_t addr = (uint32_t)__cvta_generic_to_shared(p), remote;
    int32_t v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
    return v;
}

__device__ __forceinline__ void store_remote(int32_t* p, uint32_t rank, int32_t v) {
    uint32_t addr = (uint32_t)__cvta_generic_to_shared(p), remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(remote), "r"(v) : "memory");
}

// Lets a kernel have clusters of up to 16 CTAs, once per device.
inline cudaError_t allow_large_clusters(const void* kernel) {
    static std::mutex mutex;
    static const void* known[kMaxDevices][8];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mutex);
    int i = 0;
    if (dev >= 0 && dev < kMaxDevices) {
        while (i < 8 && known[dev][i] && known[dev][i] != kernel) ++i;
        if (i < 8 && known[dev][i]) return cudaSuccess;
    }
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && dev >= 0 && dev < kMaxDevices && i < 8) known[dev][i] = kernel;
    return e;
}

template <class... P, class... A>
inline amoeba_status launch_clusters(void (*kernel)(P...), int64_t grid, int threads, size_t smem, int cluster, bool early,
                                     cudaStream_t stream, const A&... args) {
    if (smem > 16 * 1024 && ensure_dynamic_smem((const void*)kernel, (int)smem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute a[2] = {};
    if (cluster > 1) {
        a[c.numAttrs].id = cudaLaunchAttributeClusterDimension;
        a[c.numAttrs].val.clusterDim.x = (unsigned)cluster;
        a[c.numAttrs].val.clusterDim.y = a[c.numAttrs].val.clusterDim.z = 1;
        ++c.numAttrs;
    }
    if (early) {
        a[c.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        a[c.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++c.numAttrs;
    }
    c.attrs = a;
    if (cudaLaunchKernelEx(&c, kernel, static_cast<P>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return AMOEBA_ERR_CUDA;
    }
    count_launch();
    return AMOEBA_OK;
}

}  // namespace amoeba
