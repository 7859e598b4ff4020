// Verification of drafted tokens against the target's probabilities, from given random numbers (rejection sampling that keeps
// the target's distribution).  With p_i the target's and q_i the draft model's probabilities at draft i, x_i the drafted token:
//
//   draft i is kept while  u_i q_i(x_i) < p_i(x_i);  r = the first that is not (n where all are)
//   the token after the kept ones is drawn from  w = max(p_r - q_r, 0)  (r < n; p_r where that is zero everywhere)  or  w = p_n:
//   the least k with  w_0 + ... + w_k > u (w_0 + ... + w_{V-1})
//
// Everything is formed in 64 bits: the products and differences of 32-bit numbers are then exact, and the sums are off by so
// little that the order in which they are added does not show in which token is drawn.
//
// Two rows of the vocabulary a sequence are read once (one where all drafts are kept).  Bound by latency, with few sequences and with many: 128 of
// 131071 tokens take 27 us for 93 MB, 3.4 TB/s, because a warp asks for a tile when it has added up the one before.
// A cluster of CTAs shares a sequence: every warp adds up tiles of 256 tokens, the tiles' sums stay in shared memory, the CTAs' sums
// are exchanged, and the one CTA in whose part the threshold falls looks for the tile and reads that again (it is in L2).
#include <cooperative_groups.h>

#include "kvs_cache.cuh"

namespace kvs {

namespace cg = cooperative_groups;

constexpr int VER_THREADS = 256;
constexpr int VER_TILE = 256;               // tokens a warp adds up at a time: 8 loads of either row in flight a lane (512: 4 x 32000 6.6 -> 7.7 us; 1024: 128 x 131071 27 -> 42)
constexpr int VER_MOST_SMEM = 64 * 1024;    // sums of 2^21 tokens' tiles: one CTA's part up to there, beyond that of eight CTAs

struct VerifyParams {
    const float* target;        // [S, n + 1, V]
    const float* draft;         // [S, n, V]
    const int32_t* drafted;     // [S, n]
    const float* u_accept;      // [S, n]
    const float* u_sample;      // [S]
    int32_t* tokens;            // [S, n + 1]
    int32_t* n_accepted;        // [S]
    int n, V, part;             // part: tokens of a CTA, a multiple of VER_TILE
};

// weights of this lane's tokens of a tile, in 64 bits; no weight past the vocabulary, where the draft has more, or for a NaN
__device__ __forceinline__ void verify_tile(const float* p, const float* q, int k0, int V, int lane, double (&w)[VER_TILE / 32]) {
    float a[VER_TILE / 32], b[VER_TILE / 32];
    if (k0 + VER_TILE <= V && q) {               // a whole tile: all loads on their way before the first is used
#pragma unroll
        for (int i = 0; i < VER_TILE / 32; ++i) a[i] = __ldg(p + k0 + i * 32 + lane);
#pragma unroll
        for (int i = 0; i < VER_TILE / 32; ++i) b[i] = __ldg(q + k0 + i * 32 + lane);
    } else {
#pragma unroll
        for (int i = 0; i < VER_TILE / 32; ++i) {
            const int k = k0 + i * 32 + lane;
            a[i] = k < V ? __ldg(p + k) : 0.f;
            b[i] = (q && k < V) ? __ldg(q + k) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < VER_TILE / 32; ++i) w[i] = a[i] > b[i] ? (double)a[i] - (double)b[i] : 0.0;
}

__global__ void __launch_bounds__(VER_THREADS) verify_kernel(VerifyParams p) {
    extern __shared__ double s_tile[];          // sum of every tile of this CTA's part
    __shared__ double s_sum, s_warp[VER_THREADS / 32];
    __shared__ int s_kept, s_last;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
    const int s = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    // ---- how many drafts are kept (every CTA of the cluster for itself) ----
    if (warp == 0) {
        int kept = p.n;
        for (int i0 = 0; i0 < p.n && kept == p.n; i0 += 32) {
            const int i = i0 + lane;
            bool ok = true;
            if (i < p.n) {
                const int x = p.drafted[(size_t)s * p.n + i];
                ok = (unsigned)x < (unsigned)p.V;                 // a token outside the vocabulary has no probability
                if (ok) {
                    const double px = p.target[((size_t)s * (p.n + 1) + i) * p.V + x], qx = p.draft[((size_t)s * p.n + i) * p.V + x];
                    ok = (double)p.u_accept[(size_t)s * p.n + i] * qx < px;
                }
            }
            const unsigned no = __ballot_sync(0xffffffffu, !ok);
            if (no) kept = i0 + __ffs(no) - 1;
        }
        if (lane == 0) s_kept = kept;
    }
    __syncthreads();
    const int kept = s_kept;
    const float* row = p.target + ((size_t)s * (p.n + 1) + kept) * p.V;
    const float* less = kept < p.n ? p.draft + ((size_t)s * p.n + kept) * p.V : nullptr;
    const int k_begin = min(c * p.part, p.V), k_end = min(k_begin + p.part, p.V);
    const int ntiles = (k_end - k_begin + VER_TILE - 1) / VER_TILE;
    double before = 0.0, total = 0.0, mine = 0.0;
    for (int attempt = 0; attempt < 2; ++attempt) {
        for (int t = warp; t < ntiles; t += VER_THREADS / 32) {
            double w[VER_TILE / 32], sum = 0.0;
            verify_tile(row, less, k_begin + t * VER_TILE, p.V, lane, w);
#pragma unroll
            for (int i = 0; i < VER_TILE / 32; ++i) sum += w[i];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) s_tile[t] = sum;
        }
        __syncthreads();
        double sum = 0.0;
        for (int t = tid; t < ntiles; t += VER_THREADS) sum += s_tile[t];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        if (tid == 0) {
            sum = 0.0;
            for (int i = 0; i < VER_THREADS / 32; ++i) sum += s_warp[i];
            s_sum = sum;
        }
        cluster.sync();
        before = total = mine = 0.0;
        for (int i = 0; i < C; ++i) {
            const double x = *cluster.map_shared_rank(&s_sum, i);
            if (i < c) before += x;
            if (i == c) mine = x;
            total += x;
        }
        cluster.sync();                          // the sums have been read: they may be written again, or the CTA may leave
        if (total > 0.0 || !less) break;         // the same decision in the whole cluster
        less = nullptr;                          // the draft has as much everywhere: drawn from the target's own row
    }
    // ---- the token after them: the CTA in whose part the threshold falls, or with the last weight where rounding leaves none ----
    // The CTAs' parts [before, before + mine) are added up in one order everywhere, so they follow one another without a gap.
    double bar = fmin(fmax((double)p.u_sample[s], 0.0), 1.0) * total;
    if (!(bar < total)) bar = total;
    const bool here = bar < total ? before <= bar && bar < before + mine : before < total && before + mine >= total;
    if (here) {
        if (warp == 0) {
            // the tile: the first whose running sum passes the threshold; failing that the last with any weight
            int at = -1, last = 0;
            double run = before;
            for (int t0 = 0; t0 < ntiles && at < 0; t0 += 32) {
                const double x = t0 + lane < ntiles ? s_tile[t0 + lane] : 0.0;
                double y = x;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double z = __shfl_up_sync(0xffffffffu, y, o);
                    if (lane >= o) y += z;
                }
                const unsigned over = __ballot_sync(0xffffffffu, x > 0.0 && run + y > bar), some = __ballot_sync(0xffffffffu, x > 0.0);
                if (some) last = t0 + 31 - __clz(some);
                if (over) {
                    const int l = __ffs(over) - 1;
                    at = t0 + l;
                    run += __shfl_sync(0xffffffffu, y - x, l);
                } else {
                    run += __shfl_sync(0xffffffffu, y, 31);
                }
            }
            const bool passes = at >= 0;
            if (!passes) at = last;
            // the token inside it
            double w[VER_TILE / 32];
            verify_tile(row, less, k_begin + at * VER_TILE, p.V, lane, w);
            int token = -1, least = -1;
#pragma unroll
            for (int i = 0; i < VER_TILE / 32; ++i) {
                double y = w[i];
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double z = __shfl_up_sync(0xffffffffu, y, o);
                    if (lane >= o) y += z;
                }
                const unsigned over = __ballot_sync(0xffffffffu, w[i] > 0.0 && run + y > bar), some = __ballot_sync(0xffffffffu, w[i] > 0.0);
                if (some) least = i * 32 + 31 - __clz(some);
                if (over && token < 0) token = i * 32 + __ffs(over) - 1;
                run += __shfl_sync(0xffffffffu, y, 31);
            }
            if (lane == 0) s_last = k_begin + at * VER_TILE + (passes && token >= 0 ? token : least);
        }
        __syncthreads();
    }
    if (here || (total == 0.0 && c == 0)) {
        const int next = here ? s_last : -1;     // a row without any probability gives no token
        for (int i = tid; i <= p.n; i += VER_THREADS)
            p.tokens[(size_t)s * (p.n + 1) + i] = i < kept ? p.drafted[(size_t)s * p.n + i] : i == kept ? next : -1;
        if (tid == 0) p.n_accepted[s] = kept;
    }
}

}  // namespace kvs

using namespace kvs;

extern "C" int kvs_verify_drafts(const float* target_probs, const float* draft_probs, const int32_t* draft_tokens, const float* u_accept,
                                 const float* u_sample, int num_seqs, int n_draft, int vocab, int32_t* tokens, int32_t* n_accepted,
                                 kvs_stream_t stream) {
    if (num_seqs < 0 || n_draft < 0 || vocab <= 0) return KVS_ERR_INVALID_ARG;
    if (vocab > (1 << 24) || n_draft > 65535 || num_seqs > (1 << 24)) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0) return KVS_OK;
    if (!target_probs || !u_sample || !tokens || !n_accepted) return KVS_ERR_INVALID_ARG;
    if (n_draft > 0 && (!draft_probs || !draft_tokens || !u_accept)) return KVS_ERR_INVALID_ARG;
    if ((((uintptr_t)target_probs | (uintptr_t)draft_probs | (uintptr_t)draft_tokens | (uintptr_t)u_accept | (uintptr_t)u_sample | (uintptr_t)tokens |
          (uintptr_t)n_accepted) & 3) != 0)
        return KVS_ERR_ALIGNMENT;
    const int tiles = (vocab + VER_TILE - 1) / VER_TILE;
    int C = 8;
    while (C > 1 && ((long long)num_seqs * C > 4 * 148 || tiles < C)) C >>= 1;
    if (vocab > (1 << 21)) C = 8;                // the tiles' sums fit into shared memory
    VerifyParams p = {target_probs, draft_probs, draft_tokens, u_accept, u_sample, tokens, n_accepted, n_draft, vocab, (tiles + C - 1) / C * VER_TILE};
    const size_t smem = (size_t)(p.part / VER_TILE) * sizeof(double);
    // the same limit in every call: it belongs to the function, and another thread's call may come between this line and the launch
    if (smem > 40 * 1024 && cudaFuncSetAttribute(verify_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, VER_MOST_SMEM) != cudaSuccess)
        return cuda_refused();
    return launch_clusters_after(verify_kernel, dim3((unsigned)(num_seqs * C)), C, VER_THREADS, smem, (cudaStream_t)stream, p);
}
