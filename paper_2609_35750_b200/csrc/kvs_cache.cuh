// What the kernels of the rollout side share: the header of the free list, launches of clusters.
#pragma once

#include "kvs_common.cuh"

namespace kvs {

struct CacheHeader {            // the first 16 bytes of the free-list buffer
    int32_t top;                // number of free pages on the stack
    int32_t status;             // KVS_OK or an error recorded by a kernel
    int32_t refused;            // kvs_cache_append_tokens: the call in flight could not have its pages
    int32_t pad;
};

constexpr size_t DEC_WS_HEADER = 256;       // of a decode workspace: {magic, status}; the splits' results follow

// The splits of (sequence, token, query head) rows and where their merged results go
struct MergeParams {
    const float* part_o;
    const float* part_ml;
    __nv_bfloat16* out;
    float* lse;
    int32_t* header;
    int rows, nsplit;                    // nsplit: splits that there is room for
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

// The status of a call is gathered with its partial results, so that no launch of its own has to reset the workspace's word before
// any CTA may write to it: a CTA that met an error (a bad page id, a wait that ran out) hands over its sums, which are never
// negative, with the sign bit set and the kind in the lowest bit.  The first CTA writes {magic, OK}, the merge adds the errors.
__device__ __forceinline__ float flagged_sum(float sum, int status) {
    const uint32_t bits = __float_as_uint(sum) & 0x7fffffffu;
    return __uint_as_float(status == KVS_OK ? bits : (bits & ~1u) | 0x80000000u | (status == KVS_ERR_TIMEOUT ? 1u : 0u));
}
__device__ __forceinline__ float sum_and_status(float flagged, int32_t* status) {
    const uint32_t bits = __float_as_uint(flagged);
    if (bits >> 31) set_status(status, bits & 1u ? KVS_ERR_TIMEOUT : KVS_ERR_INVALID_ARG);
    return __uint_as_float(bits & 0x7fffffffu);
}
// Merge of the `count` splits (of p.nsplit that there is room for) of a (sequence, query head) by a warp: weights exp2(m_z - max), normalised, bf16 out and fp32 lse.  Bound by
// latency: the loads of PART splits are on their way before the first is used (16: with 4 at a time 47 splits took 7 us more);
// where there are few splits, PART = 4 leaves room for twice the warps (100 sequences of 64 heads, one split: step 38.0 ->
// 34.8 us).  A kernel of its own, started by programmatic dependent launch: merging in the last CTA of a (sequence, KV head) to
// finish, with counts in the workspace, cost every CTA a fence and an atomic and the merge its parallelism (a step in a CUDA
// graph, merge in the last CTA -> here, us: 1 x 24000 tokens with 8 heads on 1 29.6 -> 15.0, 1 x 2000 with 32 on 8 14.2 -> 12.7,
// 100 x 300 with 8 on 8 and head_dim 64 17.4 -> 13.5; launched call by call 30.4 -> 15.8, 14.6 -> 13.3, 17.9 -> 13.8).
template <int D, int PART>
__device__ __forceinline__ void decode_merge_row(const MergeParams& p, size_t row, int lane, int count) {
    constexpr int PER = D / 32;
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row * p.nsplit;
    const float* po = p.part_o + row * p.nsplit * D + lane * PER;
    float M = -INFINITY;
    for (int z = lane; z < count; z += 32) M = fmaxf(M, __ldcg(ml + z).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    const float Mu = (M == -INFINITY) ? 0.f : M;
    float L = 0.f, acc[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = 0.f;
    for (int z0 = 0; z0 < count; z0 += 32) {
        const float2 x = (z0 + lane < count) ? __ldcg(ml + z0 + lane) : make_float2(-INFINITY, 0.f);
        const float w = fast_exp2(x.x - Mu);
        L += sum_and_status(x.y, p.header + 1) * w;
        for (int i0 = 0; i0 < min(32, count - z0); i0 += PART) {
            float v[PART][PER];
#pragma unroll
            for (int i = 0; i < PART; ++i) {
                const float* src = po + (size_t)(z0 + i0 + i) * D;
                const bool there = z0 + i0 + i < count;
                if constexpr (PER == 4) {
                    const float4 y = there ? __ldcg(reinterpret_cast<const float4*>(src)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    v[i][0] = y.x; v[i][1] = y.y; v[i][2] = y.z; v[i][3] = y.w;
                } else {
                    const float2 y = there ? __ldcg(reinterpret_cast<const float2*>(src)) : make_float2(0.f, 0.f);
                    v[i][0] = y.x; v[i][1] = y.y;
                }
            }
#pragma unroll
            for (int i = 0; i < PART; ++i) {
                const float wi = __shfl_sync(0xffffffffu, w, i0 + i);
#pragma unroll
                for (int e = 0; e < PER; ++e) acc[e] += v[i][e] * wi;
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    const float inv = L == 0.f ? 0.f : 1.f / L;           // a NaN among the scores stays in both results
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] *= inv;
    if constexpr (PER == 4)
        *reinterpret_cast<uint2*>(p.out + row * D + lane * PER) = make_uint2(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]));
    else
        *reinterpret_cast<uint32_t*>(p.out + row * D + lane * PER) = pack_bf16(acc[0], acc[1]);
    if (lane == 0) p.lse[row] = L == 0.f ? -INFINITY : M * 0.6931471805599453f + logf(L);
}
// The row of this warp where CTAs of MERGE_WARPS warps have a row a warp.  There are up to 2^31 - 1 rows: their threads would not fit into 32 bits.
constexpr int MERGE_WARPS = 8;
__device__ __forceinline__ unsigned merge_row() { return blockIdx.x * (unsigned)MERGE_WARPS + (threadIdx.x >> 5); }
inline unsigned merge_ctas(int rows) { return ((unsigned)rows + MERGE_WARPS - 1) / MERGE_WARPS; }
// TMA gather: the 64-column slice starting at column c0 of the four rows r0..r3 of a 2-D tensor lands in four
// consecutive 128-byte rows at dst (swizzled by address like a tiled box); completes 512 bytes on the barrier.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, int c0, int r0, int r1, int r2, int r3, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar)
        : "memory");
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
