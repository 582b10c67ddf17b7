// Thread-block clusters: their blocks' shared memory, and launches.
#pragma once
#include <atomic>
#include <cstdint>

#include "common.cuh"

namespace ipotk {

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
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The two halves of a barrier: what lies between them need not wait.
__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of `p`, a pointer into this block's shared memory, in block `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 cluster_ld2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_st(uint32_t addr, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void cluster_st(uint32_t addr, float2 v) { asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory"); }
__device__ __forceinline__ void cluster_st(uint32_t addr, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory"); }

inline void cluster_config(cudaLaunchConfig_t &lc, cudaLaunchAttribute (&at)[2], dim3 grid, dim3 block, size_t smem, int cluster)
{
    lc.gridDim = grid;
    lc.blockDim = block;
    lc.dynamicSmemBytes = smem;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
}

// A launch of clusters along x, as a programmatic dependent like launch_pdl's.  More than 8 blocks a cluster (not portable, but this part has 16) have to be allowed to a kernel on
// every device that it runs on, and anew after a device's reset: at each launch, like the size of its shared memory.
constexpr int kPortableRanks = 8;
template <typename... P, typename... A>
inline cudaError_t launch_cluster(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[2];
    cluster_config(lc, at, grid, block, smem, cluster);
    lc.stream = stream;
    if (cluster > kPortableRanks) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return cudaLaunchKernelEx(&lc, kern, P(args)...);
}

// Blocks of a cluster for `items` pieces of work, each spread over one: the most, up to `most`, with which all clusters run side by side.  How many do is the driver's answer, asked once
// per kernel, device, shared memory of a block and size: the blocks of a cluster share a GPC, and with one block an SM 15 clusters of 8 fit this part, not 18.
constexpr int kMostRanks = 16;
struct ClusterFit {   // of one kernel
    static constexpr int kDevices = 16, kSizes = 8;   // (beyond these, or where two sizes share a place, it is asked again)
    std::atomic<uint64_t> seen[kDevices][kSizes][kMostRanks + 1];   // shared memory << 32 | clusters + 1; 0: not asked yet
};
template <typename Kernel>
inline int choose_cluster(ClusterFit &fit, Kernel kern, dim3 block, size_t smem, long long items, int most)
{
    int device;
    if (cudaGetDevice(&device) != cudaSuccess) {
        cudaGetLastError();
        return 1;
    }
    const uint32_t size = (uint32_t)smem * 2654435761u >> 29;
    for (int c = most < kMostRanks ? most : kMostRanks; c > 1; --c) {
        std::atomic<uint64_t> *place = device < ClusterFit::kDevices ? &fit.seen[device][size][c] : nullptr;
        const uint64_t was = place ? place->load(std::memory_order_relaxed) : 0;
        int n = (int)(was & 0xffffffffu) - 1;
        if (!was || was >> 32 != smem) {
            cudaLaunchConfig_t lc = {};
            cudaLaunchAttribute at[2];
            cluster_config(lc, at, dim3(c), block, smem, c);
            if ((c > kPortableRanks && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
                cudaOccupancyMaxActiveClusters(&n, kern, &lc) != cudaSuccess) {
                cudaGetLastError();
                n = 0;
            }
            if (place) place->store((uint64_t)smem << 32 | (uint32_t)(n + 1), std::memory_order_relaxed);
        }
        if (items <= n) return c;
    }
    return 1;
}

}  // namespace ipotk
