// The paged cache's life with accumulated attention weights and drafted tokens: the pages with the lowest weight leave, several
// tokens of every sequence join in one call, the last ones leave again.
//
// Every call is two kernels at most, and one where it is small.  The first is one CTA: it goes over the sequences' lengths, counts the
// pages that each takes or gives back, and hands every sequence its place on the free stack by a running sum, so that the order of the
// stack does not depend on which CTA comes first (the counts follow from the lengths alone, whichever pages they turn out to be).  A call
// that cannot be done for lack of pages is not begun.  The second kernel moves the data.
#include <cooperative_groups.h>

#include "kvs_cache.cuh"

namespace kvs {

namespace cg = cooperative_groups;

constexpr int PLAN_THREADS = 1024;

// of tokens >= 0; both below 2^31, so that unsigned words hold the sum
__device__ __forceinline__ int pages_of(int tokens, int page_size) { return (int)(((unsigned)tokens + (unsigned)page_size - 1u) / (unsigned)page_size); }

// ---- eviction of the lowest pages ------------------------------------------------------------------
// Score of a page: its tokens' weights added up in 64 bits, rounded to 32.  The candidates are the full pages with no token among the
// first keep_first or the last keep_recent; those with the lowest scores leave, of equal ones the earlier slots, as many as bring the
// sequence to its budget (or all of them).
//
// A cluster of CTAs shares a sequence, each with a run of its pages in shared memory (scores or weights, table).  The threshold is
// found by a radix search on the scores' order-preserving bits, 8 at a time: every CTA counts its candidates' digits, the counts are
// added over the cluster through distributed shared memory, and the digit in which the sought rank falls is fixed.  Then every page
// knows from two prefix sums (how many lie below the threshold before it, how many on it) whether it leaves and where it goes, and
// table and weights are written back in order: all reads are over before the first write.
// Bound by latency: 64 caches of 16384 to 32768 one-token pages of which half leave, 29 MB in all, take 4.5 + 22 us (floor 4.8): 3 us until
// weights and table are in shared memory, 3 for each of three digits, 7 for the ranks and the lists, 2 to write back.
constexpr int EV_THREADS = 512;
constexpr int EV_COPIES = 8;                // of the counts, by lane: scores crowd into a few digits
constexpr int EV_MOST_CTAS = 8;             // of a cluster
constexpr int EV_MOST_SMEM = 208 * 1024, EV_PLAIN_SMEM = 32 * 1024;      // dynamic, beside 11 KB; without asking for more than 48 KB

struct EvictParams {
    int budget, keep_first, keep_recent, S, page_size, max_pages, num_pages;
    int32_t* block_table;
    int32_t* n_tokens;
    int32_t* free_buf;
    float* weight;              // [S, max_pages * page_size]
    int32_t* evicted;           // [S, max_pages] or null
    int32_t* n_evicted;         // [S]
};

__device__ __forceinline__ void candidates(const EvictParams& p, int n, int& lo, int& hi) {
    lo = pages_of(p.keep_first, p.page_size);
    hi = n > p.keep_recent ? (n - p.keep_recent) / p.page_size : 0;
}
__device__ __forceinline__ int pages_to_leave(const EvictParams& p, int n) {
    int lo, hi;
    candidates(p, n, lo, hi);
    return n > p.budget ? min(pages_of(n - p.budget, p.page_size), max(0, hi - lo)) : 0;
}

__global__ void __launch_bounds__(PLAN_THREADS) evict_plan_kernel(EvictParams p) {
    __shared__ int s_warp[33];
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(p.free_buf);
    pdl_wait();
    const int top = hdr->top;
    int sum = 0, total;
    for (int s = threadIdx.x; s < p.S; s += blockDim.x) {
        const int n = p.n_tokens[s];
        if (n >= 0 && pages_of(n, p.page_size) <= p.max_pages) sum += pages_to_leave(p, n);
        else set_status(&hdr->status, KVS_ERR_INVALID_ARG);          // a length that the table cannot hold: this sequence stays as it is
    }
    block_prefix(sum, s_warp, total);
    const bool fits = top >= 0 && total <= p.num_pages - top;        // else more pages would come back than the cache has: nothing is done
    __syncthreads();
    if (threadIdx.x == 0) {
        if (fits) hdr->top = top + total;
        else set_status(&hdr->status, KVS_ERR_INVALID_ARG);
    }
    for (int s = threadIdx.x; s < p.S; s += blockDim.x) {
        const int n = p.n_tokens[s];
        const int take = fits && n >= 0 && pages_of(n, p.page_size) <= p.max_pages ? pages_to_leave(p, n) : 0;
        p.n_evicted[s] = take;
        if (take > 0) p.n_tokens[s] = n - take * p.page_size;
    }
}

// ascending in the score; -0 is 0, a NaN is above everything
__device__ __forceinline__ uint32_t score_bits(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b >> 31) ? ~b : b | 0x80000000u;
}

// TOGETHER: at most EV_MOST_CTAS sequences, each small enough for a CTA.  They are one cluster: every CTA reads all lengths and forms the
// plan itself, and nothing is written before all have, so that one launch does what takes two otherwise.  Up to what fits into shared memory
// without asking for more, and 2048 pages.  Both sides, by two launches -> by one (us, with 4.6 for the copy of the state before it): four
// caches in pages of 16: 1000 tokens 15.4 -> 10.8, 6500 16.4 -> 12.3 (the border), 10000 16.4 -> 13.4, 20000 16.7 -> 17.0, 40000 18.1 -> 24.6; in
// one-token pages: 1000 16.5 -> 10.8, 2000 16.4 -> 12.4 (the border), 4000 16.4 -> 16.4, 10000 18.5 -> 22.6; one cache or eight about the same.
template <bool TOGETHER>
__global__ void __launch_bounds__(EV_THREADS) evict_kernel(EvictParams p, int cap) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ int s_hist[2][256];               // digits of this CTA's candidates, for the cluster
    __shared__ __align__(16) int s_count[256 * EV_COPIES];
    __shared__ int s_warp[33];
    __shared__ unsigned long long s_warp64[33];
    __shared__ int s_bin, s_below, s_in_bin;
    __shared__ int2 s_counts;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = TOGETHER ? 1 : (int)cluster.num_blocks(), c = TOGETHER ? 0 : (int)cluster.block_rank();
    const int s = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31;
    const int ps = p.page_size;
    auto sync = [&]() {                          // of a sequence's CTAs
        if (TOGETHER) __syncthreads();
        else cluster.sync();
    };
    const int stride = ps | 1;                   // of a page's weights: threads that add up a page each read different banks
    float* s_w = reinterpret_cast<float*>(smem_raw);                              // [cap * stride] weights
    int32_t* s_page = reinterpret_cast<int32_t*>(s_w + (size_t)cap * stride);     // [cap] table entries
    uint16_t* s_src = reinterpret_cast<uint16_t*>(s_page + cap);                  // [cap] pages that stay, in order
    uint32_t* s_key = reinterpret_cast<uint32_t*>(s_src + ((cap + 1) & ~1));      // [cap] scores (pages of one token: formed from s_w)
    pdl_wait();
    int take, n, base;                           // pages that leave, live tokens, this sequence's place behind what those before it give back
    int32_t* stack;                              // the j-th page goes to stack[-j]
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(p.free_buf);
    if (TOGETHER) {
        // every warp for itself, a lane for a sequence
        const int top = hdr->top, ni = lane < p.S ? p.n_tokens[lane] : 0;
        const bool ok = ni >= 0 && pages_of(ni, ps) <= p.max_pages;
        const int leave = ok ? pages_to_leave(p, ni) : 0;
        const bool bad = __any_sync(0xffffffffu, !ok);
        const int total = __reduce_add_sync(0xffffffffu, leave);
        base = __reduce_add_sync(0xffffffffu, lane < s ? leave : 0);
        take = __shfl_sync(0xffffffffu, leave, s);
        n = __shfl_sync(0xffffffffu, ni, s);
        const bool fits = top >= 0 && total <= p.num_pages - top;
        if (!fits) take = 0;
        cluster.sync();                          // all have read: now it may be written
        if (tid == 0) {
            p.n_evicted[s] = take;
            if (take > 0) p.n_tokens[s] = n - take * ps;
            if (s == 0 && fits) hdr->top = top + total;
            if (s == 0 && (bad || !fits)) set_status(&hdr->status, KVS_ERR_INVALID_ARG);
        }
        stack = p.free_buf + 4 + (top + total - 1 - base);
    } else {
        take = p.n_evicted[s];
    }
    int32_t* evicted = p.evicted ? p.evicted + (size_t)s * p.max_pages : nullptr;
    if (evicted)
        for (int i = take + c * EV_THREADS + tid; i < p.max_pages; i += C * EV_THREADS) evicted[i] = -1;
    if (take <= 0) return;                               // the same in the whole cluster (TOGETHER: its CTAs do not meet again)
    if (!TOGETHER) {
        int mine = 0;
        for (int i = tid; i < s; i += EV_THREADS) mine += p.n_evicted[i];
        block_prefix(mine, s_warp, base);
        stack = p.free_buf + 4 + (hdr->top - 1 - base);
        n = p.n_tokens[s] + take * ps;
    }
    const int live = pages_of(n, ps);
    int lo, hi;
    candidates(p, n, lo, hi);
    const int per = (live + C - 1) / C, first = min(c * per, live), count = min(first + per, live) - first;
    int32_t* table = p.block_table + (size_t)s * p.max_pages;
    float* weight = p.weight + (size_t)s * p.max_pages * ps;
#pragma unroll 8
    for (int i = tid; i < count; i += EV_THREADS) s_page[i] = table[first + i];
    if (stride == ps) {
#pragma unroll 8
        for (int i = tid; i < count * ps; i += EV_THREADS) s_w[i] = weight[(size_t)first * ps + i];
    } else {
#pragma unroll 8
        for (int i = tid; i < count * ps; i += EV_THREADS) s_w[i + (int)((unsigned)i / (unsigned)ps)] = weight[(size_t)first * ps + i];
    }
    for (int i = tid; i < 256 * EV_COPIES; i += EV_THREADS) s_count[i] = 0;
    __syncthreads();
    if (ps > 1) {
        for (int i = tid; i < count; i += EV_THREADS) {
            double sum = 0.0;
            for (int j = 0; j < ps; ++j) sum += (double)s_w[i * stride + j];
            s_key[i] = score_bits((float)sum);
        }
        __syncthreads();
    }
    auto key_of = [&](int i) { return ps == 1 ? score_bits(s_w[i]) : s_key[i]; };
    const int from = max(lo - first, 0), until = min(hi - first, count);          // this CTA's candidates
    // ---- the threshold: `take` candidates are below it, or on it and early ----
    uint32_t found = 0;
    int want = take;                                     // how many of those whose upper digits are `found`
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        int* hist = s_hist[pass & 1];
#pragma unroll 4
        for (int i = from + tid; i < until; i += EV_THREADS) {
            const uint32_t key = key_of(i);
            if (pass == 0 || (key >> (shift + 8)) == (found >> (shift + 8)))
                atomicAdd(&s_count[((key >> shift) & 255u) * EV_COPIES + (lane & (EV_COPIES - 1))], 1);
        }
        __syncthreads();
        if (tid < 256) {
            int4* copies = reinterpret_cast<int4*>(s_count + tid * EV_COPIES);
            const int4 x = copies[0], y = copies[1];
            hist[tid] = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w;
            copies[0] = copies[1] = make_int4(0, 0, 0, 0);
        }
        sync();
        int sum = 0;
        if (tid < 256) {
            int part[EV_MOST_CTAS];                      // all on their way before the first is added: a remote read takes most of a microsecond
#pragma unroll
            for (int i = 0; i < EV_MOST_CTAS; ++i) part[i] = TOGETHER ? (i == 0 ? hist[tid] : 0) : i < C ? cluster.map_shared_rank(hist, i)[tid] : 0;
#pragma unroll
            for (int i = 0; i < EV_MOST_CTAS; ++i) sum += part[i];
        }
        int all;
        const int below = block_prefix(sum, s_warp, all);
        if (tid < 256 && below < want && want <= below + sum) {
            s_bin = tid;
            s_below = below;
            s_in_bin = sum;
        }
        __syncthreads();
        found |= (uint32_t)s_bin << shift;
        want -= s_below;
        if (want == s_in_bin && shift > 0) {             // everything with these digits leaves: no need to look further
            found |= (1u << shift) - 1u;
            break;
        }
        __syncthreads();
    }
    // ---- which pages leave, and where the others go ----
    const int run = (count + EV_THREADS - 1) / EV_THREADS | 1;           // odd: the threads' pages lie in different banks
    const int a = min(tid * run, count), z = min(a + run, count);
    int under = 0, on = 0;
#pragma unroll 4
    for (int i = max(a, from); i < min(z, until); ++i) {
        const uint32_t key = key_of(i);
        under += key < found;
        on += key == found;
    }
    unsigned long long both;                             // the two counts side by side
    const unsigned long long before = block_prefix((unsigned long long)under << 32 | (unsigned)on, s_warp64, both);
    const int under_all = (int)(both >> 32), on_all = (int)(both & 0xffffffffu);
    int under_before = (int)(before >> 32), on_before = (int)(before & 0xffffffffu);
    if (tid == 0) s_counts = make_int2(under_all, on_all);
    sync();
    int under_first = 0, on_first = 0, on_total = 0, under_total = 0;
    int2 other[EV_MOST_CTAS];
#pragma unroll
    for (int i = 0; i < EV_MOST_CTAS; ++i) other[i] = TOGETHER ? (i == 0 ? s_counts : make_int2(0, 0)) : i < C ? *cluster.map_shared_rank(&s_counts, i) : make_int2(0, 0);
#pragma unroll
    for (int i = 0; i < EV_MOST_CTAS; ++i) {
        if (i < c) {
            under_first += other[i].x;
            on_first += other[i].y;
        }
        under_total += other[i].x;
        on_total += other[i].y;
    }
    const int of_equals = min(take - under_total, on_total);     // of those on the threshold the earlier slots leave
    under_before += under_first;
    on_before += on_first;
    const int gone_first = under_first + min(on_first, of_equals);
    for (int i = a; i < z; ++i) {
        bool leaves = false;
        const int rank = under_before + min(on_before, of_equals);
        if (i >= from && i < until) {
            const uint32_t key = key_of(i);
            if (key < found) {
                leaves = true;
                ++under_before;
            } else if (key == found) {
                leaves = on_before < of_equals;
                ++on_before;
            }
        }
        // pages that stay from the front of the list, pages that leave from its end
        s_src[leaves ? count - 1 - (rank - gone_first) : i - (rank - gone_first)] = (uint16_t)i;
    }
    __syncthreads();
    const int gone_here = under_all + min(on_first + on_all, of_equals) - min(on_first, of_equals);
    const int stays = count - gone_here, to = first - gone_first;        // page k that stays goes to slot `to + k`
    for (int k = tid; k < gone_here; k += EV_THREADS) {
        const int src = s_src[count - 1 - k];
        stack[-(gone_first + k)] = s_page[src];
        if (evicted) evicted[gone_first + k] = first + src;
    }
    for (int k = tid; k < stays; k += EV_THREADS) {
        const int src = s_src[k];
        if (to + k != first + src) table[to + k] = s_page[src];
    }
    if (ps == 1) {
        for (int k = tid; k < stays; k += EV_THREADS) {
            const int src = s_src[k];
            if (to + k != first + src) weight[to + k] = s_w[src];
        }
    } else for (int i = tid; i < stays * ps; i += EV_THREADS) {
        const int k = (int)((unsigned)i / (unsigned)ps), src = s_src[k];
        if (to + k != first + src) weight[(size_t)to * ps + i] = s_w[src * stride + (i - k * ps)];
    }
    // no weight behind the last page
    for (int i = (live - take) * ps + c * EV_THREADS + tid; i < live * ps; i += C * EV_THREADS) weight[i] = 0.f;
    if (!TOGETHER) cluster.sync();                       // the others have read this CTA's counts
}

// ---- several tokens of every sequence join --------------------------------------------------------------
struct JoinParams {
    const __nv_bfloat16* k_new;        // [S, n_new, Hkv, D]
    const __nv_bfloat16* v_new;
    const uint8_t* active;             // [S] or null
    int S, n_new, row, page_size, max_pages, num_pages;          // row: elements of a token, Hkv * D
    int32_t* block_table;
    int32_t* n_tokens;
    int32_t* free_buf;
    __nv_bfloat16* k_cache;
    __nv_bfloat16* v_cache;
};

// Why a call is not begun, whichever sequence is looked at first: a state that makes no sense comes before a want of room.
__device__ __forceinline__ int join_refusal(const JoinParams& p, bool senseless, bool full, int top, int total) {
    if (senseless || top < 0 || top > p.num_pages) return KVS_ERR_INVALID_ARG;
    return full || total > top ? KVS_ERR_WORKSPACE : KVS_OK;
}

// One CTA: pages for the new tokens of all sequences, or of none.  The j-th page of the call comes from stack[top - 1 - j].
__global__ void __launch_bounds__(PLAN_THREADS) join_plan_kernel(JoinParams p) {
    __shared__ int s_warp[33];
    __shared__ bool s_senseless, s_full;                 // set by any thread, cleared by none
    __shared__ int s_n[PLAN_THREADS], s_at[PLAN_THREADS];
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(p.free_buf);
    const int32_t* stack = p.free_buf + 4;
    const int tid = threadIdx.x;
    if (tid == 0) s_senseless = s_full = false;
    __syncthreads();
    pdl_wait();
    auto joins = [&](int s) { return s < p.S && (!p.active || p.active[s]); };
    auto needs = [&](int n) { return pages_of(n + p.n_new, p.page_size) - pages_of(n, p.page_size); };
    const int top = hdr->top;
    int sum = 0, total;
    for (int s = tid; s < p.S; s += blockDim.x) {
        if (!joins(s)) continue;
        const int n = p.n_tokens[s];
        const long long room = (long long)p.max_pages * p.page_size;
        if (n < 0 || n > room) s_senseless = true;
        else if (n > room - p.n_new) s_full = true;
        else sum += needs(n);
    }
    block_prefix(sum, s_warp, total);                    // its synchronisations order the two words too
    const int no = join_refusal(p, s_senseless, s_full, top, total);
    __syncthreads();
    if (tid == 0) {
        hdr->refused = no != KVS_OK;
        if (no == KVS_OK) hdr->top = top - total;
        else set_status(&hdr->status, no);
    }
    if (no != KVS_OK) return;                            // the same in the whole CTA
    int base = 0;
    for (int s0 = 0; s0 < p.S; s0 += blockDim.x) {
        const int s = s0 + tid;
        const bool in = joins(s);
        const int n = in ? p.n_tokens[s] : 0, need = in ? needs(n) : 0;
        int here;
        s_at[tid] = base + block_prefix(need, s_warp, here);
        s_n[tid] = in ? n : -1;
        base += here;
        if (in) p.n_tokens[s] = n + p.n_new;
        __syncthreads();
        for (int i = tid >> 5; i < min((int)blockDim.x, p.S - s0); i += blockDim.x / 32) {        // a warp for a sequence
            if (s_n[i] < 0) continue;
            const int slot = pages_of(s_n[i], p.page_size), pages = needs(s_n[i]);
            for (int j = tid & 31; j < pages; j += 32)
                p.block_table[(size_t)(s0 + i) * p.max_pages + slot + j] = stack[top - 1 - (s_at[i] + j)];
        }
        __syncthreads();
    }
}

// Few rows: both steps in one launch, by one cluster.  Every CTA forms the plan itself and nothing is written before all have read; a new
// page's number comes from the stack and not from the table, which the first CTA fills in meanwhile.
constexpr int JOIN_CTAS = 8, JOIN_THREADS = 512, JOIN_SEQS = 128;
template <typename T>
__global__ void __launch_bounds__(JOIN_THREADS) join_together_kernel(JoinParams p) {
    __shared__ int s_warp[33];
    __shared__ bool s_senseless, s_full;                 // set by any thread, cleared by none
    __shared__ int s_n[JOIN_SEQS], s_at[JOIN_SEQS];
    cg::cluster_group cluster = cg::this_cluster();
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(p.free_buf);
    const int32_t* stack = p.free_buf + 4;
    const int tid = threadIdx.x, c = (int)cluster.block_rank();
    constexpr int PER = sizeof(T) / sizeof(__nv_bfloat16);
    const int words = p.row / PER;
    if (tid == 0) s_senseless = s_full = false;
    __syncthreads();
    pdl_wait();
    const int top = hdr->top;
    int need = 0, total;
    if (tid < JOIN_SEQS) {
        const bool in = tid < p.S && (!p.active || p.active[tid]);
        const int n = in ? p.n_tokens[tid] : 0;
        const long long room = (long long)p.max_pages * p.page_size;
        if (n < 0 || n > room) s_senseless = true;
        else if (in && n > room - p.n_new) s_full = true;
        else if (in) need = pages_of(n + p.n_new, p.page_size) - pages_of(n, p.page_size);
        s_n[tid] = in ? n : -1;
    }
    const int at = block_prefix(need, s_warp, total);
    if (tid < JOIN_SEQS) s_at[tid] = at;
    const int no = join_refusal(p, s_senseless, s_full, top, total);
    cluster.sync();                                      // all have read: now it may be written (and the sums are in place)
    if (c == 0 && tid == 0) {
        hdr->refused = no != KVS_OK;
        if (no == KVS_OK) hdr->top = top - total;
        else set_status(&hdr->status, no);
    }
    if (no != KVS_OK) return;                            // the same in the whole cluster
    if (c == 0 && tid < p.S && s_n[tid] >= 0) {
        p.n_tokens[tid] = s_n[tid] + p.n_new;
        const int slot = pages_of(s_n[tid], p.page_size);
        for (int j = 0; j < need; ++j) p.block_table[(size_t)tid * p.max_pages + slot + j] = stack[top - 1 - (at + j)];
    }
    const int items = p.S * p.n_new * words;
    for (int i = c * JOIN_THREADS + tid; i < items; i += JOIN_CTAS * JOIN_THREADS) {
        const int token = i / words, w = i - token * words, s = token / p.n_new;
        if (s_n[s] < 0) continue;
        const int pos = s_n[s] + (token - s * p.n_new), slot = pos / p.page_size, fresh = slot - pages_of(s_n[s], p.page_size);
        const T k = reinterpret_cast<const T*>(p.k_new)[i], v = reinterpret_cast<const T*>(p.v_new)[i];
        const int page = fresh >= 0 ? stack[top - 1 - (s_at[s] + fresh)] : p.block_table[(size_t)s * p.max_pages + slot];
        if ((unsigned)page >= (unsigned)p.num_pages) {               // an entry that names no page of this cache is not followed
            set_status(&hdr->status, KVS_ERR_INVALID_ARG);
            continue;
        }
        const size_t dst = ((size_t)page * p.page_size + (pos - slot * p.page_size)) * words + w;
        reinterpret_cast<T*>(p.k_cache)[dst] = k;
        reinterpret_cast<T*>(p.v_cache)[dst] = v;
    }
}

// The rows: T is what is copied at a time (16 bytes, or an element where rows are no multiple of that).
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(JoinParams p) {
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(p.free_buf);
    constexpr int PER = sizeof(T) / sizeof(__nv_bfloat16);
    const int words = p.row / PER;
    pdl_wait();
    if (hdr->refused) return;
    const long long items = (long long)p.S * p.n_new * words;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long long)gridDim.x * 256) {
        const long long token = i / words;
        const int w = (int)(i - token * words), s = (int)(token / p.n_new), t = (int)(token - (long long)s * p.n_new);
        if (p.active && !p.active[s]) continue;
        const int at = p.n_tokens[s] - p.n_new + t, slot = at / p.page_size;
        const T k = reinterpret_cast<const T*>(p.k_new)[i], v = reinterpret_cast<const T*>(p.v_new)[i];
        const int page = p.block_table[(size_t)s * p.max_pages + slot];
        if ((unsigned)page >= (unsigned)p.num_pages) {               // an entry that names no page of this cache is not followed
            set_status(&hdr->status, KVS_ERR_INVALID_ARG);
            continue;
        }
        const size_t dst = ((size_t)page * p.page_size + (at - slot * p.page_size)) * words + w;
        reinterpret_cast<T*>(p.k_cache)[dst] = k;
        reinterpret_cast<T*>(p.v_cache)[dst] = v;
    }
}

// ---- the last tokens leave -------------------------------------------------------------------------------
// One CTA: sequence s loses its last n_drafted - n_accepted[s] tokens.  Pages go back in the order that undoes kvs_cache_append_tokens:
// the j-th of the call to stack[top + total - 1 - j].
__global__ void __launch_bounds__(PLAN_THREADS) truncate_kernel(int n_drafted, const int32_t* __restrict__ n_accepted, int S, int page_size, int max_pages,
                                                                int num_pages, const int32_t* __restrict__ block_table, int32_t* n_tokens, int32_t* free_buf,
                                                                float* weight) {
    __shared__ int s_warp[33];
    __shared__ int s_from[PLAN_THREADS], s_to[PLAN_THREADS], s_at[PLAN_THREADS];
    CacheHeader* hdr = reinterpret_cast<CacheHeader*>(free_buf);
    int32_t* stack = free_buf + 4;
    const int tid = threadIdx.x;
    pdl_wait();
    // tokens that leave; none where the counts make no sense
    auto leaves = [&](int s, int n, bool tell) {
        const int kept = n_accepted[s];
        if (n < 0 || pages_of(n, page_size) > max_pages || kept < 0 || kept > n_drafted || n_drafted - kept > n) {
            if (tell) set_status(&hdr->status, KVS_ERR_INVALID_ARG);
            return 0;
        }
        return n_drafted - kept;
    };
    const int top = hdr->top;
    int sum = 0, total;
    for (int s = tid; s < S; s += blockDim.x) {
        const int n = n_tokens[s], gone = leaves(s, n, true);
        sum += gone > 0 ? pages_of(n, page_size) - pages_of(n - gone, page_size) : 0;
    }
    block_prefix(sum, s_warp, total);
    const bool fits = top >= 0 && total <= num_pages - top;
    __syncthreads();
    if (tid == 0) {
        if (fits) hdr->top = top + total;
        else set_status(&hdr->status, KVS_ERR_INVALID_ARG);
    }
    if (!fits) return;                                   // the same in the whole CTA
    int base = 0;
    for (int s0 = 0; s0 < S; s0 += blockDim.x) {
        const int s = s0 + tid, n = s < S ? n_tokens[s] : 0, gone = s < S ? leaves(s, n, false) : 0;
        const int pages = gone > 0 ? pages_of(n, page_size) - pages_of(n - gone, page_size) : 0;
        int here;
        s_at[tid] = base + block_prefix(pages, s_warp, here);
        s_from[tid] = n - gone;
        s_to[tid] = n;
        base += here;
        if (gone > 0) n_tokens[s] = n - gone;
        __syncthreads();
        for (int i = tid >> 5; i < min((int)blockDim.x, S - s0); i += blockDim.x / 32) {          // a warp for a sequence
            if (s_from[i] >= s_to[i]) continue;
            const int slot = pages_of(s_from[i], page_size), end = pages_of(s_to[i], page_size);
            for (int j = tid & 31; j < end - slot; j += 32)
                stack[top + total - 1 - (s_at[i] + j)] = block_table[(size_t)(s0 + i) * max_pages + slot + j];
            if (weight)
                for (int t = s_from[i] + (tid & 31); t < s_to[i]; t += 32) weight[(size_t)(s0 + i) * max_pages * page_size + t] = 0.f;
        }
        __syncthreads();
    }
}

}  // namespace kvs

using namespace kvs;

// A thread for a sequence, and a warp for its pages: few sequences need no large CTA
static int plan_threads(int num_seqs, bool warps) {
    const int want = warps ? num_seqs * 32 : num_seqs;
    return want <= 128 ? 128 : want <= 256 ? 256 : want <= 512 ? 512 : PLAN_THREADS;
}
// Tokens of a sequence and pages of all sequences are counted in 32 bits: a sum that wrapped would pass for one that fits the stack
static bool counts_fit(int num_seqs, int page_size, int max_pages) {
    return (long long)max_pages * page_size <= 0x7fffffffLL && (long long)num_seqs * max_pages <= 0x7fffffffLL;
}
static bool cache_sizes_ok(int num_seqs, int page_size, int max_pages, int num_pages) {
    return num_seqs >= 0 && page_size > 0 && max_pages > 0 && num_pages > 0;
}

extern "C" int kvs_cache_evict_lowest(int budget, int keep_first, int keep_recent, int num_seqs, int page_size, int max_pages, int num_pages,
                                      int32_t* block_table, int32_t* n_tokens, int32_t* free_list, float* token_weight, int32_t* evicted,
                                      int32_t* n_evicted, kvs_stream_t stream) {
    if (!cache_sizes_ok(num_seqs, page_size, max_pages, num_pages) || budget < 0 || keep_first < 0 || keep_recent < 0) return KVS_ERR_INVALID_ARG;
    if (num_seqs > (1 << 24) || !counts_fit(num_seqs, page_size, max_pages)) return KVS_ERR_UNSUPPORTED;
    // the cluster holds a sequence's weights, table and scores in shared memory
    const long long page_bytes = 4ll * (page_size | 1) + 6 + (page_size > 1 ? 4 : 0);
    int C = 1;
    // more CTAs where a sequence has more than 1024 tokens for each and two CTAs an SM are not yet taken, or where it does not fit
    while (C < EV_MOST_CTAS && (((long long)max_pages * page_size > 1024ll * C && (long long)num_seqs * C < 148) ||
                                ((long long)(max_pages + C - 1) / C + 2) * page_bytes > EV_MOST_SMEM))
        C <<= 1;
    const int cap = (max_pages + C - 1) / C;
    const size_t smem = (size_t)((cap + 2) * page_bytes);
    if (smem > EV_MOST_SMEM || cap > 65535) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0) return KVS_OK;
    if (!block_table || !n_tokens || !free_list || !token_weight || !n_evicted) return KVS_ERR_INVALID_ARG;
    if ((((uintptr_t)block_table | (uintptr_t)n_tokens | (uintptr_t)free_list | (uintptr_t)token_weight | (uintptr_t)evicted | (uintptr_t)n_evicted) & 3) != 0)
        return KVS_ERR_ALIGNMENT;
    const EvictParams p = {budget, keep_first, keep_recent, num_seqs, page_size, max_pages, num_pages, block_table, n_tokens, free_list, token_weight, evicted,
                           n_evicted};
    cudaStream_t st = (cudaStream_t)stream;
    const size_t alone = (size_t)((max_pages + 2) * page_bytes);
    if (num_seqs <= EV_MOST_CTAS && max_pages <= 2048 && alone <= EV_PLAIN_SMEM)
        return launch_clusters_after(evict_kernel<true>, dim3((unsigned)num_seqs), num_seqs, EV_THREADS, alone, st, p, max_pages);
    // the same limit in every call: it belongs to the function, and another thread's call may come between this line and the launch
    if (smem > EV_PLAIN_SMEM && cudaFuncSetAttribute(evict_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_MOST_SMEM) != cudaSuccess)
        return cuda_refused();
    const int rc = launch_after(evict_plan_kernel, 1, plan_threads(num_seqs, false), 0, st, p);
    if (rc != KVS_OK) return rc;
    return launch_clusters_after(evict_kernel<false>, dim3((unsigned)(num_seqs * C)), C, EV_THREADS, smem, st, p, cap);
}

extern "C" int kvs_cache_append_tokens(const void* k_new, const void* v_new, const uint8_t* active, int num_seqs, int n_new, int Hkv, int head_dim,
                                       int page_size, int max_pages, int num_pages, int32_t* block_table, int32_t* n_tokens, int32_t* free_list,
                                       void* k_cache, void* v_cache, kvs_stream_t stream) {
    if (!cache_sizes_ok(num_seqs, page_size, max_pages, num_pages) || n_new < 0 || Hkv <= 0 || head_dim <= 0) return KVS_ERR_INVALID_ARG;
    if (!counts_fit(num_seqs, page_size, max_pages) || (long long)Hkv * head_dim > 0x7fffffffLL) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0 || n_new == 0) return KVS_OK;
    if (!k_new || !v_new || !block_table || !n_tokens || !free_list || !k_cache || !v_cache) return KVS_ERR_INVALID_ARG;
    const uintptr_t rows = (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)k_cache | (uintptr_t)v_cache;
    if ((rows & 1) != 0 || (((uintptr_t)block_table | (uintptr_t)n_tokens | (uintptr_t)free_list) & 3) != 0) return KVS_ERR_ALIGNMENT;
    const JoinParams p = {(const __nv_bfloat16*)k_new, (const __nv_bfloat16*)v_new, active, num_seqs, n_new, Hkv * head_dim, page_size, max_pages, num_pages,
                          block_table, n_tokens, free_list, (__nv_bfloat16*)k_cache, (__nv_bfloat16*)v_cache};
    cudaStream_t st = (cudaStream_t)stream;
    const bool wide = (p.row % 8) == 0 && (rows & 15) == 0;
    const long long items = (long long)num_seqs * n_new * (wide ? p.row / 8 : p.row);
    // the cluster has 4096 threads: up to four words each they are faster than a second launch (append and truncate: 4 x 4 tokens 6.2 -> 5.3 us,
    // 16 x 5 7.8 -> 7.3, 128 x 1 12.1 -> 9.7; at eight words a thread both take 7.6)
    if (num_seqs <= JOIN_SEQS && items <= 4 * JOIN_CTAS * JOIN_THREADS)
        return wide ? launch_clusters_after(join_together_kernel<uint4>, JOIN_CTAS, JOIN_CTAS, JOIN_THREADS, 0, st, p)
                    : launch_clusters_after(join_together_kernel<uint16_t>, JOIN_CTAS, JOIN_CTAS, JOIN_THREADS, 0, st, p);
    const int rc = launch_after(join_plan_kernel, 1, plan_threads(num_seqs, true), 0, st, p);
    if (rc != KVS_OK) return rc;
    const unsigned grid = (unsigned)((items + 255) / 256 < 148 * 8 ? (items + 255) / 256 : 148 * 8);
    return wide ? launch_after(join_kernel<uint4>, grid, 256, 0, st, p) : launch_after(join_kernel<uint16_t>, grid, 256, 0, st, p);
}

extern "C" int kvs_cache_truncate(int n_drafted, const int32_t* n_accepted, int num_seqs, int page_size, int max_pages, int num_pages,
                                  const int32_t* block_table, int32_t* n_tokens, int32_t* free_list, float* token_weight, kvs_stream_t stream) {
    if (!cache_sizes_ok(num_seqs, page_size, max_pages, num_pages) || n_drafted < 0) return KVS_ERR_INVALID_ARG;
    if (!counts_fit(num_seqs, page_size, max_pages)) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0 || n_drafted == 0) return KVS_OK;
    if (!n_accepted || !block_table || !n_tokens || !free_list) return KVS_ERR_INVALID_ARG;
    if ((((uintptr_t)n_accepted | (uintptr_t)block_table | (uintptr_t)n_tokens | (uintptr_t)free_list | (uintptr_t)token_weight) & 3) != 0)
        return KVS_ERR_ALIGNMENT;
    return launch_after(truncate_kernel, 1, plan_threads(num_seqs, true), 0, (cudaStream_t)stream, n_drafted, n_accepted, num_seqs, page_size, max_pages, num_pages, block_table,
                        n_tokens, free_list, token_weight);
}
