// Attention of the last n_new live tokens of every sequence over its paged cache, with a sliding window and a few first tokens that
// stay visible.  Query t stands at p = n - n_new + t; it sees live token j iff  j <= p and (j < sinks or j > p - window).
//
// Bound by HBM: the K and V rows that any of the queries sees are read once, tiles and pages that none sees are not touched.  Both
// products run on the tensor core in the transposed form, so that a tile's 128 keys fill its 128 rows and the few queries its columns:
//   S^T [128 keys x N] = K [128 x d] Q^T            A = K tile, B = Q: column c is query head c % G of token c / G
//   O^T [d x N]       += V^T [d x 128 keys] P^T     A = V tile read MN-major, B = P^T  (d = 64: rows 64 .. 127 repeat rows 0 .. 63)
// One CTA per (split, KV head, sequence and group of new tokens): four softmax warps (a thread has a key of S^T and a column d of
// O^T) and a control warp (block table, TMA loads, MMA issue).  K of tile t + 1 is asked for as soon as S^T of tile t is complete, V of
// tile t as soon as the second product of tile t - 1 is; two or three CTAs an SM overlap one another's loads, products and softmax.
// Rows reach shared memory as in kvs_decode_attn: pages of 8 to 128 tokens that tile 128 by one TMA box each, others by rows (K by
// TMA gather4, V by cp.async).
//
// The softmax needs no maximum in most tiles: weights are taken against a reference per column in shared memory, a tile goes on
// with it while no score is more than 2^8 above (one barrier that also takes a vote), and only else the columns' maxima are formed, the
// reference moves and O^T is rescaled.
//
// A tile in which some query does not see some key is masked by element.  V rows that no query sees are cleared in shared memory
// (0 x NaN is NaN).  A V row that some see and others do not (the new tokens, the window's edge) may hold an infinity or a NaN: it is
// cleared too and added by hand for the queries that see it (`patch`).
#include <cstring>

#include "kvs_cache.cuh"

namespace kvs {
__device__ long long g_cta[8192*8];
__device__ __forceinline__ long long gt() { long long t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
__device__ __forceinline__ int smid() { int t; asm volatile("mov.u32 %0, %smid;" : "=r"(t)); return t; }
#define CT(i) if (lin < 8192 && threadIdx.x == 0) g_cta[lin * 8 + (i)] = gt();

constexpr int WIN_THREADS = 160;
constexpr int WIN_PAGES = 1;         // one TMA box per page
constexpr int WIN_ROWS = 2;          // K: TMA gather4; V: cp.async rows
constexpr float WIN_UNSET = -1e30f;  // reference of a column that has seen no key yet: any score is far above it

struct WindowParams {
    const __nv_bfloat16* q;          // [S, n_new, Hq, D]
    const __nv_bfloat16* v_cache;    // [num_pages, page_size, Hkv, D]
    const int32_t* block_table;      // [S, max_pages]
    const int32_t* n_tokens;         // [S]
    int S, n_new, Hq, Hkv, G, page_size, page_shift, max_pages, num_pages, nsplit;
    int groups, group_tokens;        // new tokens of a sequence in groups of group_tokens: G * group_tokens columns at most
    int window, sinks;
    int32_t* header;
    float scale_log2;
    float* part_o;                   // [S * n_new * Hq, nsplit, D] unnormalised
    float* part_ml;                  // [S * n_new * Hq, nsplit, 2]
};

template <int D, int COLS>
struct WinSmem {
    static constexpr int TILE_BYTES = 128 * D * 2;
    static constexpr int OFF_K = 0;
    static constexpr int OFF_V = TILE_BYTES;
    static constexpr int OFF_Q = 2 * TILE_BYTES;                       // [COLS x D] bf16, boxes of 64 columns
    static constexpr int OFF_P = OFF_Q + COLS * D * 2;                 // P^T as [COLS x 128 keys] bf16, two boxes of 64 keys
    static constexpr int OFF_BAR = OFF_P + COLS * 256;
    static constexpr int OFF_MISC = OFF_BAR + 64;                      // tmem base, abort flag, status, bad rows of the tile before
    static constexpr int OFF_REF = OFF_MISC + 64;                      // [COLS] reference, base-2 units
    static constexpr int OFF_AT = OFF_REF + COLS * 4;                  // [COLS] position of the column's token
    static constexpr int OFF_ROW = OFF_AT + COLS * 4;                  // [COLS] its row among all (sequence, token, query head)
    static constexpr int OFF_ALPHA = OFF_ROW + COLS * 4;               // [COLS]
    static constexpr int OFF_WMAX = OFF_ALPHA + COLS * 4;              // [4 warps][COLS]
    static constexpr int TOTAL = OFF_WMAX + COLS * 16;
    static constexpr int DYN_BYTES = TOTAL + 1024;                     // slack for the 1024-byte alignment
};

__device__ __forceinline__ int window_order(float x) {                 // order-preserving map float -> int
    const int i = __float_as_int(x);
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float window_unorder(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }
// Whether any thread of the group says so, the same answer for each
__device__ __forceinline__ bool group_any(int id, int nthreads, bool mine) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %3, 0;\n\t"
        "bar.red.or.pred q, %1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"(id), "r"(nthreads), "r"((uint32_t)mine)
        : "memory");
    return any != 0;
}

template <int D, int COLS, int LOAD>
__global__ void __launch_bounds__(WIN_THREADS, COLS <= 16 || (COLS <= 32 && D == 64) ? 3 : 2)
decode_window_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ WindowParams p) {
    using SM = WinSmem<D, COLS>;
    constexpr int BOX = 16384, NBOX = D / 64;
    constexpr int QBOX = COLS * 128;                     // bytes of a 64-wide box of Q or P^T
    constexpr uint32_t IDESC_S = make_idesc(COLS, 0, 0), IDESC_O = make_idesc(COLS, 1, 0);
    constexpr bool PAGES = LOAD == WIN_PAGES;
    extern __shared__ uint8_t smem_raw[];
    const int z = blockIdx.x, g = blockIdx.y, s = blockIdx.z / p.groups, group = blockIdx.z - s * p.groups;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int lin = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
    CT(0)
    pdl_wait();
    CT(1)

    if ((blockIdx.x | blockIdx.y | blockIdx.z | threadIdx.x) == 0) {
        p.header[0] = (int32_t)WS_MAGIC;
        p.header[1] = KVS_OK;
    }
    const int ps = p.page_size, G = p.G;
    const int n = min(max(p.n_tokens[s], 0), p.max_pages * ps);          // never past the sequence's table
    const int tok0 = group * p.group_tokens, ntok = min(p.group_tokens, p.n_new - tok0), cols = ntok * G;
    // positions of the group's queries: at0 .. end - 1 (negative ones see nothing); keys below `head` or in [lo, end) are seen by some
    const int at0 = n - p.n_new + tok0, end = max(at0 + ntok, 0);
    const int head = min(p.sinks, end);
    const int lo = max(0, max(at0, 0) - (p.window - 1));
    const int head_tiles = (head + 127) >> 7, body = max(lo >> 7, head_tiles);
    const int all_tiles = head_tiles + max(0, ((end + 127) >> 7) - body);
    const int per = (all_tiles + p.nsplit - 1) / p.nsplit;               // contiguous tiles per split
    const int i_begin = min(z * per, all_tiles), my_tiles = min(i_begin + per, all_tiles) - i_begin;
    auto tile_at = [&](int i) { return i_begin + i < head_tiles ? i_begin + i : body + (i_begin + i - head_tiles); };
    auto seen_by_some = [&](int j) { return j < head || (j >= lo && j < end); };

    const uint32_t sraw = smem_u32(smem_raw), sbase = (sraw + 1023u) & ~1023u;
    uint8_t* sgen = smem_raw + (sbase - sraw);
    const uint32_t sK = sbase + SM::OFF_K, sV = sbase + SM::OFF_V, sQ = sbase + SM::OFF_Q, sP = sbase + SM::OFF_P, bars = sbase + SM::OFF_BAR;
    // as in the decode kernel: K / V rows have landed, S^T complete (hence K, and the V and P^T of the tile before, consumed), P^T
    // written, second product complete
    const uint32_t bar_kfull = bars, bar_vfull = bars + 8, bar_s = bars + 16, bar_p = bars + 24, bar_done = bars + 32;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(sgen + SM::OFF_MISC);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sgen + SM::OFF_MISC + 4);
    int32_t* status = reinterpret_cast<int32_t*>(sgen + SM::OFF_MISC + 8);
    volatile uint32_t* s_bad = reinterpret_cast<volatile uint32_t*>(sgen + SM::OFF_MISC + 16);           // [4]
    float* s_ref = reinterpret_cast<float*>(sgen + SM::OFF_REF);
    int* s_at = reinterpret_cast<int*>(sgen + SM::OFF_AT);
    int* s_row = reinterpret_cast<int*>(sgen + SM::OFF_ROW);
    float* s_alpha = reinterpret_cast<float*>(sgen + SM::OFF_ALPHA);
    float* s_wmax = reinterpret_cast<float*>(sgen + SM::OFF_WMAX);

    if (tid == 0) {
        *abort_flag = 0;
        *status = KVS_OK;
        mbar_init(bar_kfull, 1);
        mbar_init(bar_vfull, 1);
        mbar_init(bar_s, 1);
        mbar_init(bar_p, 128);
        mbar_init(bar_done, 1);
        fence_mbar_init();
    }
    if (warp == 4) {
        tmem_alloc(smem_u32(s_tmem), 2 * COLS);
        tmem_relinquish();
    } else {
        if (tid < COLS) {
            const int t = tid / G;
            s_ref[tid] = tid < cols ? WIN_UNSET : 0.f;       // columns past the last score 0 and never move
            s_at[tid] = tid < cols ? at0 + t : -1;
            s_row[tid] = tid < cols ? (s * p.n_new + tok0 + t) * p.Hq + g * G + (tid - t * G) : -1;
        }
        named_bar_sync(1, 128);
        // column c, 16-byte chunk of its row: box, then chunk ^ (c % 8) of the 128-byte row; columns past the last are zero
        constexpr int NQ = COLS * (D / 8) / 128;             // chunks a thread, all on their way before the first is stored
        uint4 v[NQ];
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            const int i = tid + k * 128, row = s_row[i / (D / 8)];
            v[k] = row >= 0 ? *reinterpret_cast<const uint4*>(p.q + (size_t)row * D + (i % (D / 8)) * 8) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            const int i = tid + k * 128, c = i / (D / 8), c16 = i % (D / 8);
            *reinterpret_cast<uint4*>(sgen + SM::OFF_Q + (c16 >> 3) * QBOX + c * 128 + (((c16 & 7) ^ (c & 7)) << 4)) = v[k];
        }
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    CT(2)
    const uint32_t tmem_S = *s_tmem, tmem_O = tmem_S + COLS;
    const int32_t* bt = p.block_table + (size_t)s * p.max_pages;
    auto split_token = [&](int tok, int& entry, int& offset) {
        entry = p.page_shift >= 0 ? tok >> p.page_shift : tok / ps;
        offset = tok - entry * ps;
    };
    // an entry that names no page of the cache is recorded and read as page 0
    auto checked_page = [&](int page) {
        if ((unsigned)page < (unsigned)p.num_pages) return page;
        set_status(status, KVS_ERR_INVALID_ARG);
        return 0;
    };

    if (warp == 4) {
        // ================= control warp: block table, TMA loads, MMA issue =================
        const bool leader = elect_one();
        const uint64_t dK = smem_desc(sK, 16, 1024), dQ = smem_desc(sQ, 16, 1024);
        const uint64_t dV = smem_desc(sV, D == 128 ? BOX : 0, 1024), dP = smem_desc(sP, 16, 1024);
        const int ppt = PAGES ? 128 / ps : 0;                  // pages per tile
        // PAGES: lane i has page i of the tile, if some query sees a row of it; ROWS: lane L the pages of rows 4 L .. 4 L + 3 (rows past the
        // end repeat the last one: their scores are masked), if some query sees one of them
        struct Ids { int v[PAGES ? 1 : 4]; bool need; };
        auto fetch_ids = [&](int i, Ids& id) {
            id.need = false;
            if (i >= my_tiles) return;
            const int k0 = tile_at(i) * 128;
            const int a = k0 + lane * (PAGES ? ps : 4), e = min(a + (PAGES ? ps : 4), end);
            id.need = (!PAGES || lane < ppt) && a < e && (a < head || e > lo);
            if (PAGES) {
                id.v[0] = id.need ? bt[tile_at(i) * ppt + lane] : 0;
            } else if (id.need) {
#pragma unroll
                for (int j = 0; j < (PAGES ? 1 : 4); ++j) {
                    int en, o;
                    split_token(min(a + j, end - 1), en, o);
                    id.v[j] = bt[en];
                }
            }
        };
        auto load_pages = [&](const CUtensorMap* map, uint32_t dst, uint32_t bar, const Ids& id) {
            const uint32_t pages = __popc(__ballot_sync(0xffffffffu, id.need));
            if (leader) mbar_expect_tx(bar, pages * (uint32_t)(ps * D * 2));
            __syncwarp();
            if (id.need) {
                const int row = checked_page(id.v[0]) * ps;
#pragma unroll
                for (int b = 0; b < NBOX; ++b) tma_load_3d(dst + b * BOX + (uint32_t)(lane * ps) * 128u, map, b * 64, g, row, bar);
            }
        };
        auto load_k = [&](int i, const Ids& id) {              // K buffer must be free
            if constexpr (PAGES) {
                load_pages(&tm_k, sK, bar_kfull, id);
            } else {
                const uint32_t quads = __popc(__ballot_sync(0xffffffffu, id.need));
                if (leader) mbar_expect_tx(bar_kfull, quads * (uint32_t)(4 * D * 2));
                __syncwarp();
                if (id.need) {
                    int row[4];
    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int en, o;
                        split_token(min(tile_at(i) * 128 + 4 * lane + j, end - 1), en, o);
                        row[j] = checked_page(id.v[j]) * ps + o;
                    }
    #pragma unroll
                    for (int b = 0; b < NBOX; ++b) tma_gather4(sK + b * BOX + (uint32_t)lane * 512u, &tm_k, g * D + b * 64, row[0], row[1], row[2], row[3], bar_kfull);
                }
            }
        };
        Ids cur, nxt;
        for (int j = 0; j < (PAGES ? 1 : 4); ++j) cur.v[j] = nxt.v[j] = 0;
        fetch_ids(0, cur);
        fetch_ids(1, nxt);
        if (my_tiles > 0) load_k(0, cur);
        for (int it = 0; it < my_tiles; ++it) {
            mbar_wait(bar_kfull, it & 1, abort_flag, status);
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {          // S^T = K Q^T, 16 elements of d per step
                const uint64_t offk = (uint64_t)(((kk >> 2) * BOX + (kk & 3) * 32) >> 4);
                const uint64_t offq = (uint64_t)(((kk >> 2) * QBOX + (kk & 3) * 32) >> 4);
                if (leader) mma_ss(tmem_S, dK + offk, dQ + offq, IDESC_S, kk > 0);
            }
            if (leader) mma_commit(bar_s);
            mbar_wait(bar_s, it & 1, abort_flag, status);      // K is consumed; so are V and P^T of the tile before
            if (PAGES) load_pages(&tm_v, sV, bar_vfull, cur);
            if (it + 1 < my_tiles) load_k(it + 1, nxt);
            cur = nxt;
            fetch_ids(it + 2, nxt);
            mbar_wait(bar_p, it & 1, abort_flag, status);
            if (PAGES) mbar_wait(bar_vfull, it & 1, abort_flag, status);
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {               // O^T += V^T P^T, 16 keys per step
                const uint64_t offp = (uint64_t)(((kk >> 2) * QBOX + (kk & 3) * 32) >> 4);
                if (leader) mma_ss(tmem_O, dV + (uint64_t)(kk * 128), dP + offp, IDESC_O, (it > 0) || (kk > 0));
            }
            if (leader) mma_commit(bar_done);
        }
    } else {
        // ================= softmax warps =================
        const uint32_t lane_sel = (uint32_t)(warp * 32) << 16;
        float l_part[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) l_part[c] = 0.f;
        auto sees = [&](int j, int at) { return j <= at && (j < p.sinks || at - j < p.window); };
        // WIN_ROWS: this thread's rows of a tile's V (16 bytes of every RPI-th), the block-table entries one tile ahead; rows that no query
        // sees are filled with zeros
        constexpr int LPR = D / 8, RPI = 32 / LPR, NIT = PAGES ? 1 : 32 / RPI;
        int pid[NIT];
        auto row_of = [&](int j) { return warp * 32 + j * RPI + lane / LPR; };
        auto fetch_pids = [&](int i) {
            if constexpr (!PAGES) {
                if (i >= my_tiles) return;
#pragma unroll
                for (int j = 0; j < NIT; ++j) {
                    int en, o;
                    split_token(min(tile_at(i) * 128 + row_of(j), end - 1), en, o);
                    pid[j] = bt[en];
                }
            }
        };
        auto load_v_rows = [&](int k0) {
            const int c = lane % LPR;
#pragma unroll
            for (int j = 0; j < NIT; ++j) {
                const int r = row_of(j);
                int en, o;
                split_token(min(k0 + r, end - 1), en, o);
                const size_t row = (size_t)checked_page(pid[j]) * ps + o;
                const uint32_t dst = (uint32_t)((c >> 3) * BOX + r * 128 + (((c & 7) ^ (r & 7)) << 4)), bytes = seen_by_some(k0 + r) ? 16u : 0u;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sV + dst), "l"(p.v_cache + (row * p.Hkv + g) * D + c * 8), "r"(bytes)
                             : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // O^T += weight x V for the rows of the tile at k0 that were kept out of the second product.  O^T is up to date, P^T still there.
        auto patch = [&](int k0) {
            for (int r0 = 0; r0 < 128; r0 += 32)
                for (uint32_t m = s_bad[r0 >> 5]; m; m &= m - 1) {
                    const int r = r0 + __ffs(m) - 1;
                    int en, o;
                    split_token(k0 + r, en, o);
                    const size_t row = (size_t)checked_page(bt[en]) * ps + o;
                    const float v = __bfloat162float(p.v_cache[(row * p.Hkv + g) * D + tid % D]);
                    for (int c0 = 0; c0 < cols; c0 += 16) {
                        uint32_t x[16];
                        tmem_ld16(tmem_O + c0 + lane_sel, x);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            if (sees(k0 + r, s_at[c0 + c])) {
                                const uint8_t* w = sgen + SM::OFF_P + (r >> 6) * QBOX + (c0 + c) * 128 + ((((r & 63) >> 3) ^ (c & 7)) << 4) + ((r & 7) << 1);
                                x[c] = __float_as_uint(__uint_as_float(x[c]) + __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(w)) * v);
                            }
                        tmem_st16(tmem_O + c0 + lane_sel, x);
                        tmem_wait_st();
                    }
                }
        };
        bool to_patch = false;
        fetch_pids(0);
        for (int it = 0; it < my_tiles; ++it) {
            const int k0 = tile_at(it) * 128, j = k0 + tid;
            mbar_wait(bar_s, it & 1, abort_flag, status);       // S^T ready; V, P^T free; O^T up to date
            tc_fence_after();
            if (to_patch) {                                     // the same decision in every thread
                patch(tile_at(it - 1) * 128);
                named_bar_sync(1, 128);                         // P^T is written again below
            }
            if (!PAGES) {
                load_v_rows(k0);
                fetch_pids(it + 1);
            }
            // some query does not see some key of the tile
            const bool masked = k0 + 127 > at0 || !(k0 + 127 < p.sinks || end - 1 - k0 < p.window);
            float sc[COLS];
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += 16)
                if (c0 < cols) {
                    uint32_t r[16];
                    tmem_ld16(tmem_S + c0 + lane_sel, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; ++c) sc[c0 + c] = __uint_as_float(r[c]) * p.scale_log2;
                }
            // in blocks of 8 columns, without a branch inside, so that a block's loads and exponentials overlap
            if (masked) {
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 8)
                    if (c0 < cols) {
#pragma unroll
                        for (int c = c0; c < c0 + 8; ++c) sc[c] = sees(j, s_at[c]) ? sc[c] : -INFINITY;
                    }
            }
            bool above = false;
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += 8)
                if (c0 < cols) {
                    const float4 a = *reinterpret_cast<const float4*>(s_ref + c0), b = *reinterpret_cast<const float4*>(s_ref + c0 + 4);
                    const float ref[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int c = 0; c < 8; ++c) above |= sc[c0 + c] - ref[c] > 8.0f;
                }
            if (group_any(1, 128, above)) {
                // the columns' maxima over the tile; the references that are too low move there
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 8)
                    if (c0 < cols) {
#pragma unroll
                        for (int c = c0; c < c0 + 8; ++c) {
                            const int m = __reduce_max_sync(0xffffffffu, window_order(sc[c]));
                            if (lane == 0) s_wmax[warp * COLS + c] = window_unorder(m);
                        }
                    }
                named_bar_sync(1, 128);
                if (tid < cols) {
                    const float top = fmaxf(fmaxf(s_wmax[tid], s_wmax[COLS + tid]), fmaxf(s_wmax[2 * COLS + tid], s_wmax[3 * COLS + tid]));
                    const float ref = s_ref[tid], to = top - ref > 8.0f ? top : ref;
                    s_alpha[tid] = fast_exp2(ref - to);
                    s_ref[tid] = to;
                }
                named_bar_sync(1, 128);
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 8)
                    if (c0 < cols) {
#pragma unroll
                        for (int c = c0; c < c0 + 8; ++c) l_part[c] *= c < cols ? s_alpha[c] : 1.f;
                    }
                if (it > 0) {                     // O^T row d = tid
                    for (int c0 = 0; c0 < cols; c0 += 16) {
                        uint32_t o[16];
                        tmem_ld16(tmem_O + c0 + lane_sel, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * (c0 + c < cols ? s_alpha[c0 + c] : 0.f));
                        tmem_st16(tmem_O + c0 + lane_sel, o);
                        tmem_wait_st();
                    }
                }
            }
            // weights of key tid -> P^T[c][tid] (bf16), row c of box tid / 64
            uint8_t* prow = sgen + SM::OFF_P + (tid >> 6) * QBOX + ((tid & 7) << 1);
            const int chunk = (tid & 63) >> 3;
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += 8)
                if (c0 < cols) {
                    const float4 a = *reinterpret_cast<const float4*>(s_ref + c0), b = *reinterpret_cast<const float4*>(s_ref + c0 + 4);
                    const float ref[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float w = fast_exp2(sc[c0 + c] - ref[c]);
                        l_part[c0 + c] += w;
                        *reinterpret_cast<__nv_bfloat16*>(prow + (c0 + c) * 128 + ((chunk ^ c) << 4)) = __float2bfloat16(w);
                    }
                }
            if (!PAGES) asm volatile("cp.async.wait_group 0;" ::: "memory");
            to_patch = false;
            if (masked) {                         // the same decision in every thread
                if (PAGES) mbar_wait(bar_vfull, it & 1, abort_flag, status);
                else named_bar_sync(1, 128);      // other threads fetched this thread's row
                bool clear = !seen_by_some(j), bad = false;
                uint4* vrow = reinterpret_cast<uint4*>(sgen + SM::OFF_V + tid * 128);
                if (!clear && !(sees(j, at0) && sees(j, end - 1))) {
                    // some see it and others do not (or may not): it has to be finite
#pragma unroll
                    for (int b = 0; b < NBOX; ++b)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint4 x = vrow[b * (BOX / 16) + i];
                            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
                        }
                }
                const uint32_t bads = __ballot_sync(0xffffffffu, bad);
                if (lane == 0) s_bad[warp] = bads;
                if (clear || bad) {
#pragma unroll
                    for (int b = 0; b < NBOX; ++b)
#pragma unroll
                        for (int i = 0; i < 8; ++i) vrow[b * (BOX / 16) + i] = make_uint4(0, 0, 0, 0);
                }
                to_patch = group_any(1, 128, bad);
            }
            fence_proxy_async();      // P^T and the V rows written by this thread visible to the tensor core's reads of shared memory
            tc_fence_before();
            mbar_arrive(bar_p);
        }
        CT(3)
        // ---- this split's partial result: O^T (unnormalised), the references and the sums ----
        if (my_tiles > 0) {
            mbar_wait(bar_done, (my_tiles - 1) & 1, abort_flag, status);
            tc_fence_after();
            if (to_patch) patch(tile_at(my_tiles - 1) * 128);
        }
        // sums of 8 columns over the warp's lanes: the lanes halve the columns that they hold three times, then add twice
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += 8)
            if (c0 < cols) {
                float v[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = l_part[c0 + c];
#pragma unroll
                for (int half = 4; half > 0; half >>= 1) {
                    const bool upper = lane & (half * 4);
#pragma unroll
                    for (int c = 0; c < half; ++c) {
                        const float mine = upper ? v[c + half] : v[c], other = upper ? v[c] : v[c + half];
                        v[c] = mine + __shfl_xor_sync(0xffffffffu, other, half * 4);
                    }
                }
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
                if ((lane & 3) == 0) s_wmax[warp * COLS + c0 + (lane >> 2)] = v[0];
            }
        for (int c0 = 0; c0 < cols; c0 += 16) {
            uint32_t o[16];
            if (my_tiles > 0) {
                tmem_ld16(tmem_O + c0 + lane_sel, o);
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int c = 0; c < 16; ++c) o[c] = 0u;
            }
            if (tid < D) {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const int row = s_row[c0 + c];
                    if (row >= 0) p.part_o[((size_t)row * p.nsplit + z) * D + tid] = __uint_as_float(o[c]);
                }
            }
        }
        named_bar_sync(1, 128);
        if (tid < cols) {
            const float ref = s_ref[tid];
            float* ml = p.part_ml + ((size_t)s_row[tid] * p.nsplit + z) * 2;
            ml[0] = ref == WIN_UNSET ? -INFINITY : ref;
            ml[1] = flagged_sum(s_wmax[tid] + s_wmax[COLS + tid] + s_wmax[2 * COLS + tid] + s_wmax[3 * COLS + tid], *(volatile int32_t*)status);
        }
    }
    tc_fence_before();
    __syncthreads();
    CT(4)
    if (lin < 8192 && tid == 0) { g_cta[lin*8+5] = smid(); g_cta[lin*8+6] = my_tiles; }
    if (warp == 4) {
        __syncwarp();
        tmem_dealloc(tmem_S, 2 * COLS);
    }
}

}  // namespace kvs

using namespace kvs;

namespace {
constexpr int WIN_MOST_COLS = 64;

// Most tiles that a sequence's queries visit
long long window_tiles(int n_new, int max_tokens, int window, int sinks) {
    const long long all = ((long long)max_tokens + 127) / 128, some = ((long long)sinks + 127) / 128 + ((long long)window + n_new + 126) / 128 + 1;
    return all < some ? all : some;
}
int window_groups(int G, int n_new) {
    const int most = WIN_MOST_COLS / G;
    return (n_new + most - 1) / most;
}

template <int D, int COLS>
int launch_window(const CUtensorMap& tk, const CUtensorMap& tv, const WindowParams& p, bool pages, cudaStream_t st) {
    auto kern = pages ? decode_window_kernel<D, COLS, WIN_PAGES> : decode_window_kernel<D, COLS, WIN_ROWS>;
    constexpr int bytes = WinSmem<D, COLS>::DYN_BYTES;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return cuda_refused();
    return launch_after(kern, dim3((unsigned)p.nsplit, (unsigned)p.Hkv, (unsigned)(p.S * p.groups)), WIN_THREADS, bytes, st, tk, tv, p);
}
template <int D>
int launch_window_cols(const CUtensorMap& tk, const CUtensorMap& tv, const WindowParams& p, bool pages, cudaStream_t st) {
    const int cols = p.G * p.group_tokens;
    if (cols <= 16) return launch_window<D, 16>(tk, tv, p, pages, st);
    if (cols <= 32) return launch_window<D, 32>(tk, tv, p, pages, st);
    return launch_window<D, 64>(tk, tv, p, pages, st);
}
}  // namespace

extern "C" int kvs_decode_window_num_splits(int num_seqs, int n_new, int Hq, int Hkv, int max_tokens, int window, int sinks) {
    if (num_seqs <= 0 || n_new <= 0 || Hq <= 0 || Hkv <= 0 || max_tokens <= 0 || window <= 0 || sinks < 0) return 1;
    if (Hq % Hkv != 0 || Hq / Hkv > WIN_MOST_COLS) return 1;
    const long long tiles = window_tiles(n_new, max_tokens, window, sinks);
    const long long seqs = (long long)num_seqs * window_groups(Hq / Hkv, n_new);
    return kvs_decode_num_splits((int)(seqs < 65535 ? seqs : 65535), Hkv, (int)(tiles * 128 < 0x7fffffff ? tiles * 128 : 0x7fffffff));
}

extern "C" int kvs_decode_attn_window(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* n_tokens,
                                      int num_seqs, int n_new, int Hq, int Hkv, int head_dim, int page_size, int max_pages, int num_pages, float softmax_scale,
                                      int window, int sinks, int num_splits, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                      kvs_stream_t stream) {
    if (num_seqs < 0 || n_new < 0 || Hq <= 0 || Hkv <= 0 || page_size <= 0 || max_pages <= 0 || num_pages <= 0 || num_splits <= 0 || window <= 0 || sinks < 0)
        return KVS_ERR_INVALID_ARG;
    if (softmax_scale < 0.f || softmax_scale != softmax_scale) return KVS_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return KVS_ERR_UNSUPPORTED;
    if (Hq % Hkv != 0 || Hkv > 65535 || Hq / Hkv > WIN_MOST_COLS) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0 || n_new == 0) return KVS_OK;
    const int G = Hq / Hkv, groups = window_groups(G, n_new);
    if ((long long)num_seqs * groups > 65535 || (long long)num_seqs * n_new * Hq > 0x7fffffffLL) return KVS_ERR_UNSUPPORTED;
    if ((long long)num_pages * page_size > 0x7fffffffLL || (long long)max_pages * page_size > 0x7fffff00LL || (long long)Hkv * head_dim > 0x7fffffffLL)
        return KVS_ERR_UNSUPPORTED;
    if (!q || !k_cache || !v_cache || !block_table || !n_tokens || !out || !lse || !workspace) return KVS_ERR_INVALID_ARG;
    if ((((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15) != 0 || ((uintptr_t)workspace & 255) != 0 ||
        (((uintptr_t)block_table | (uintptr_t)n_tokens | (uintptr_t)lse) & 3) != 0)
        return KVS_ERR_ALIGNMENT;
    if (workspace_bytes < kvs_decode_workspace_bytes(num_seqs * n_new, Hq, head_dim, num_splits)) return KVS_ERR_WORKSPACE;
    int rc = check_device_sm100();
    if (rc != KVS_OK) return rc;
    WindowParams p;
    p.q = (const __nv_bfloat16*)q;
    p.v_cache = (const __nv_bfloat16*)v_cache;
    p.block_table = block_table;
    p.n_tokens = n_tokens;
    p.S = num_seqs;
    p.n_new = n_new;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.G = G;
    p.page_size = page_size;
    p.page_shift = (page_size & (page_size - 1)) == 0 ? __builtin_ctz((unsigned)page_size) : -1;
    p.max_pages = max_pages;
    p.num_pages = num_pages;
    p.nsplit = num_splits;
    p.groups = groups;
    p.group_tokens = (n_new + groups - 1) / groups;
    p.window = window;
    p.sinks = sinks;
    p.header = (int32_t*)workspace;
    p.scale_log2 = (softmax_scale == 0.f ? 1.0f / sqrtf((float)head_dim) : softmax_scale) * 1.4426950408889634f;
    p.part_o = (float*)((char*)workspace + DEC_WS_HEADER);
    p.part_ml = p.part_o + (size_t)num_seqs * n_new * Hq * num_splits * head_dim;
    // pages that are whole 8-row swizzle atoms and tile 128 tokens come by one TMA box each; no box reaches past the cache
    const bool pages = page_size % 8 == 0 && page_size <= 128 && 128 % page_size == 0;
    CUtensorMap tk, tv;
    memset(&tk, 0, sizeof(tk));
    memset(&tv, 0, sizeof(tv));
    if (pages) {
        if ((rc = make_tmap_thd(&tk, k_cache, num_pages * page_size, Hkv, head_dim, page_size)) != KVS_OK) return rc;
        if ((rc = make_tmap_thd(&tv, v_cache, num_pages * page_size, Hkv, head_dim, page_size)) != KVS_OK) return rc;
    } else {
        if ((rc = make_tmap_rows(&tk, k_cache, num_pages * page_size, Hkv * head_dim)) != KVS_OK) return rc;
    }
    cudaStream_t st = (cudaStream_t)stream;
    rc = head_dim == 64 ? launch_window_cols<64>(tk, tv, p, pages, st) : launch_window_cols<128>(tk, tv, p, pages, st);
    if (rc != KVS_OK) return rc;
    const MergeParams m = {p.part_o, p.part_ml, (__nv_bfloat16*)out, lse, p.header, num_seqs * n_new * Hq, num_splits};
    return launch_decode_merge(m, head_dim, st);
}

extern "C" void probe_read(long long* h) { cudaDeviceSynchronize(); cudaMemcpyFromSymbol(h, kvs::g_cta, sizeof(long long) * 8192*8); }
