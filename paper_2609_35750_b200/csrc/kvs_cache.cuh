// What the kernels of the rollout side share: the header of the free list, launches of clusters.
#pragma once

#include "kvs_common.cuh"

namespace kvs {

struct CacheHeader {            // the first 16 bytes of the free-list buffer
    int32_t top;                // number of free pages on the stack
    int32_t status;             // KVS_OK or an error recorded by a kernel
    int32_t joined;             // kvs_cache_append_tokens: whether the tokens of the call in flight have their pages
    int32_t pad;
};

#ifdef __CUDACC__
// launch_after with clusters of `cluster` CTAs along x
template <typename... P, typename... A>
inline int launch_clusters_after(void (*kernel)(P...), dim3 grid, int cluster, int threads, size_t smem, cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess ? KVS_OK : cuda_refused();
}

// Sum of `v` over the CTA's threads before this one (a whole number of warps, 32 at most); `total`: over all of them.  s_warp: 33 entries.
template <typename T>
__device__ __forceinline__ T block_prefix(T v, T* s_warp, T& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    T x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        const T w = lane < warps ? s_warp[lane] : T(0);
        T z = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T y = __shfl_up_sync(0xffffffffu, z, o);
            if (lane >= o) z += y;
        }
        __syncwarp();
        s_warp[lane] = z - w;
        if (lane == 31) s_warp[32] = z;
    }
    __syncthreads();
    total = s_warp[32];
    const T before = s_warp[warp] + x - v;
    __syncthreads();
    return before;
}
#endif

}  // namespace kvs
