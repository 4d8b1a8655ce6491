// Clusters of CTAs: launch, barrier, reads of a neighbour's shared memory.
#pragma once
#include "common.cuh"

__device__ __forceinline__ int vtk_cluster_rank()
{
    int r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ int vtk_cluster_size()
{
    int n;
    asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(n));
    return n;
}
// all threads of all CTAs of the cluster; what they wrote to shared memory before is visible behind it
__device__ __forceinline__ void vtk_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
// the same variable in the shared memory of CTA `rank` of the cluster
template <typename T>
__device__ __forceinline__ T vtk_cluster_read(const T *mine, int rank)
{
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "words");
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    if (sizeof(T) == 4) {
        uint32_t w;
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(w) : "r"(there) : "memory");
        return *reinterpret_cast<T *>(&w);
    }
    uint64_t w;
    asm volatile("ld.shared::cluster.b64 %0, [%1];" : "=l"(w) : "r"(there) : "memory");
    return *reinterpret_cast<T *>(&w);
}

// vtk_launch_dependent with clusters of `size` CTAs (grid a multiple of it)
template <typename... P, typename... A>
inline cudaError_t vtk_launch_clusters(const vtoken_ctx *ctx, void (*kernel)(P...), int size, dim3 grid, dim3 block, size_t smem,
                                       cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctx->cfg.plain_launches ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
