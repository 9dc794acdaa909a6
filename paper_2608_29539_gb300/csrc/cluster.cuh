// cluster.cuh -- thread-block clusters: a CTA's place, the barrier, and reads of
// another CTA's shared memory.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace logo {

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

// All threads of the cluster; shared memory written before is seen after.
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// The word at `p` (this CTA's address) in the CTA of the given rank.
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank)
{
    uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(p)), remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    return remote;
}

__device__ __forceinline__ unsigned long long cluster_read(const unsigned long long* p, uint32_t rank)
{
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_addr(p, rank)) : "memory");
    return v;
}

__device__ __forceinline__ int cluster_read(const int* p, uint32_t rank)
{
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr(p, rank)) : "memory");
    return v;
}

__device__ __forceinline__ int4 cluster_read4(const int* p, uint32_t rank)
{
    int4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(cluster_addr(p, rank))
                 : "memory");
    return v;
}

// Launch configuration of `blocks` CTAs in clusters of cs (attr: storage for the
// attribute, which the configuration points to).
inline cudaLaunchConfig_t cluster_config(unsigned blocks, unsigned threads, unsigned cs, size_t smem, cudaStream_t st,
                                         cudaLaunchAttribute* attr)
{
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = cs;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cs > 1 ? 1 : 0;  // (a launch without attributes is cheaper for the host)
    return cfg;
}

}  // namespace logo
