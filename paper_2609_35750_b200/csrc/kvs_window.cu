// Attention of the last n_new live tokens of every sequence over its paged cache, with a sliding window and a few first tokens that
// stay visible.  Query t stands at p = n - n_new + t; it sees live token j iff  j <= p and (j < sinks or j > p - window).
//
// Bound by HBM: the K and V rows that any of the queries sees are read once, tiles and pages that none sees are not touched.  Both
// products run on the tensor core in the transposed form, so that a tile's 128 keys fill its 128 rows and the few queries its columns:
//   S^T [128 keys x N] = K [128 x d] Q^T            A = K tile, B = Q: column c is query head c % G of token c / G
//   O^T [d x N]       += V^T [d x 128 keys] P^T     A = V tile read MN-major, B = P^T  (d = 64: rows 64 .. 127 repeat rows 0 .. 63)
// Four softmax warps (a thread has a key of S^T and a column d of O^T; from 17 columns on eight, each with half of the 32 or 64 that the
// kernel is compiled for: of 35 columns four warps have 32 and four 3), a warp that issues the products, one that loads K and two that load V (by one control warp a tile took 5900 clocks, 1300 of them to issue its 16 TMA
// instructions for K, as many for V; rows of 256 bytes take seven).  S^T of tile t + 1 is formed while tile t is in work; with a single buffer K
// of tile t + 2 is asked for as soon as that is complete, V of tile t + 1 as soon as the second product of tile t is, and two CTAs an SM
// overlap what is left of the chain; up to 16 columns two or three buffers do that (see `STAGES`).
//
// Every CTA has an equal share of all tiles: the tiles of (sequence and group of new tokens, KV head) follow one another, CTA c has
// tiles c share .. (c + 1) share - 1 of them, whose heads end where they end.  Lengths are ragged and known on the device alone, so every
// CTA adds them up itself; the first one leaves the sums for the merge, which finds from them which CTAs had a row.  K and V of the next
// head are on their way while the last one's result is written.  Fixed number of CTAs a sequence -> equal shares (us): one sequence with a
// window of 256 14.1 -> 10.4, 16 of 500 to 6000 tokens with 5 new ones (with append and truncate) 70 -> 66, 24 of 3000 to 16000 the same.
//
// Whole calls on caches that are not in L2: 64 sequences, 32 heads on 8, window 4096: 1.06 GB in 174 us, 6.1 TB/s (0.93 of the measured copy
// rate; 171 where calls follow one another on the same caches); nothing hidden, 48 sequences of up to 16000 tokens: 261 us, 0.98; 64 of 7000
// one-token pages, 28 heads on 4: 156 us, 0.9.  Heads of 64 have tiles of half the bytes and the same chain: 64 of 8000 to 16000 tokens, 16
// heads on 4, 166 us, 0.72, by one-token pages 159.  With 35 columns (5 new tokens, 7 heads a KV head) 0.47 GB in 97 us, 0.73 (92 on the same
// caches): 10 us until the first tile is through (launch, lengths, queries, first maxima), 12 between the first and the last CTA's end.
// With more than 16 columns 80 registers a thread do not suffice: 80 to 188 bytes a thread are spilled, by 16 columns none.
//
// Rows reach shared memory as in kvs_decode_attn: pages of 8 to 128 tokens that tile 128 by one TMA box each, others by rows (K by
// TMA gather4, V by cp.async).
//
// The softmax needs no maximum in most tiles: weights are taken against a reference per column in shared memory, which may lie anywhere
// near the scores, because bf16 has the exponents of fp32 and a weight's 8 bits are the same at any size.  A tile goes on with it while no
// score is more than 8 (in base-2 units) above, and a head begins with 7 where all scores of its first tile lie within 15 of 0: one
// barrier that also takes a vote.  Only else the columns' maxima are formed, the reference moves to 7 above them and O^T is rescaled.  So
// weights are at most 2^8, as in kvs_decode_attn (V may be as large), and a column's largest at least 2^-22 (products with V of 2^-104 still count).
//
// A tile in which some query does not see some key is masked by element.  V rows that no query sees are cleared in shared memory
// (0 x NaN is NaN).  A V row that some see and others do not (the new tokens, the window's edge) may hold an infinity or a NaN: it is
// cleared too and added by hand for the queries that see it (`patch`).
#include <cfloat>
#include <cstring>

#include "kvs_cache.cuh"

namespace kvs {

constexpr int WIN_PAGES = 1;         // one TMA box per page
constexpr int WIN_ROWS = 2;          // K: TMA gather4; V: cp.async rows
constexpr float WIN_UNSET = -FLT_MAX;  // reference of a column that has seen no key yet: any score is far above it, and a hidden key's -inf below it
constexpr float WIN_OVER = 8.f;      // a score may be that much above its column's reference: weights of up to 2^8, sums of up to 2^8 x keys x |v|
constexpr float WIN_AHEAD = 7.f;     // a reference is set that much above the scores it is set for, so that it need not move for the next larger one

struct WindowEntry {                 // of the workspace, written by the first CTA
    long long before;                // tiles of the entries before it, for one KV head
    int tiles, pad;
};
constexpr int WIN_SHARE_WORD = 2;    // the share, behind {magic, status} of the workspace's header

struct WindowParams {
    const __nv_bfloat16* q;          // [S, n_new, Hq, D]
    const __nv_bfloat16* v_cache;    // [num_pages, page_size, Hkv, D]
    const int32_t* block_table;      // [S, max_pages]
    const int32_t* n_tokens;         // [S]
    int S, n_new, Hq, Hkv, G, page_size, page_shift, max_pages, num_pages, nsplit;
    int groups, group_tokens;        // new tokens of a sequence in groups of group_tokens: G * group_tokens columns at most
    WindowEntry* entries;            // [S * groups], for the merge
    int window, sinks;
    int32_t* header;
    float scale_log2;
    float* part_o;                   // [S * n_new * Hq, nsplit, D] unnormalised
    float* part_ml;                  // [S * n_new * Hq, nsplit, 2]
};

// The tiles of a group of new tokens (entry e = sequence * groups + group), for one KV head.  Queries stand at at0 .. end - 1 (negative
// ones see nothing); keys below `head` or in [lo, end) are seen by some of them.
struct WindowUnit {
    int s, tok0, cols, at0, end, head, lo, head_tiles, body, tiles;
    __device__ __forceinline__ void load(const WindowParams& p, int e) {
        s = e / p.groups;
        const int group = e - s * p.groups, n = min(max(p.n_tokens[s], 0), p.max_pages * p.page_size);       // never past the sequence's table
        tok0 = group * p.group_tokens;
        const int ntok = min(p.group_tokens, p.n_new - tok0);
        cols = ntok * p.G;
        at0 = n - p.n_new + tok0;
        end = max(at0 + ntok, 0);
        head = min(p.sinks, end);
        lo = max(0, max(at0, 0) - (p.window - 1));
        head_tiles = (head + 127) >> 7;
        body = max(lo >> 7, head_tiles);
        tiles = head_tiles + max(0, ((end + 127) >> 7) - body);
    }
    __device__ __forceinline__ int key_of(int i) const { return (i < head_tiles ? i : body + (i - head_tiles)) * 128; }      // first key of tile i
    __device__ __forceinline__ bool seen_by_some(int j) const { return j < head || (j >= lo && j < end); }
};
// A CTA's way through its share
struct WindowCursor {
    int e, g, i;                     // entry, KV head, tile
    long long before;                // tiles of the entries before, for one KV head
    WindowUnit u;
    // to the first tile of the next head (or entry with any tile)
    __device__ __forceinline__ void next_unit(const WindowParams& p) {
        i = 0;
        if (++g < p.Hkv) return;
        g = 0;
        do {
            before += u.tiles;
            u.load(p, ++e);
        } while (u.tiles == 0);
    }
    __device__ __forceinline__ void next(const WindowParams& p) {
        if (++i == u.tiles) next_unit(p);
    }
};

template <int D, int COLS, int LOAD>
struct WinSmem {
    static constexpr int HALVES = COLS >= 32 ? 2 : 1;                  // threads that share a key's columns
    // warps beside them: one issues the products, the others load.  Issuing a tile's 64 gathers of K takes a warp 5600 clocks, twice the tile's
    // share of the memory's time: rows of 256 bytes are loaded by seven warps of one CTA where registers allow it
    static constexpr bool MANY = LOAD == WIN_ROWS && COLS <= 16 && D == 128;
    static constexpr int K_WARPS = MANY ? 3 : 1, V_WARPS = MANY ? 4 : 2, CONTROLS = 32 * (1 + K_WARPS + V_WARPS);
    static constexpr int WORKERS = 128 * HALVES, THREADS = WORKERS + CONTROLS;
    static constexpr int CTAS = COLS <= 16 && !MANY ? 3 : 2;           // that registers allow an SM: 24 warps, 80 a thread at launch ...
    static constexpr int WORKER_REGS = COLS <= 16 ? 104 : 96;          // ... and shared out among the warp groups like this
    static constexpr int CONTROL_REGS = MANY ? 64 : COLS <= 16 ? 56 : 48;
    static_assert(WORKERS * WORKER_REGS + CONTROLS * CONTROL_REGS <= THREADS * 80, "no more than the block was launched with");
    // CTAs an SM, and buffers of K and of V.  With TMA boxes and up to 16 columns one CTA with three of each keeps as much in flight as three with
    // one, and an SM's second CTA starts 5 us after its first, the third 8 (us, d = 128: 64 sequences with a window of 4096 three CTAs 177, two
    // 172.6, one 167.4; 8 of 1000 to 2000 tokens 20.2, 20.2, 18.4).  Heads of 64 have tiles of half the bytes: two CTAs with two of each (64 of
    // 8000 to 16000 tokens, 16 heads on 4: one with three 181, two with three 171, three with one 170, two with two 164; with 20 columns two with
    // one 182, two with two 171; one-token pages, three with one 176, three with two 159).  From 17 columns on the
    // softmax of one CTA is the bound (64 of 1000 to 2000 tokens with 20 columns: two with one 87, one with three 101), and rows come too
    // slowly by the warps of one (82 -> 141).
    static constexpr int RESIDENT = MANY ? 1 : LOAD == WIN_PAGES && COLS <= 16 ? (D == 128 ? 1 : 2) : CTAS;
    static constexpr int STAGES = D == 64 ? 2 : COLS <= 16 ? 3 : 1;
    static constexpr int TILE_BYTES = 128 * D * 2;
    static constexpr int OFF_K = 0;
    static constexpr int OFF_V = STAGES * TILE_BYTES;
    static constexpr int OFF_Q = 2 * STAGES * TILE_BYTES;              // [COLS x D] bf16, boxes of 64 columns
    static constexpr int OFF_P = OFF_Q + COLS * D * 2;                 // P^T as [COLS x 128 keys] bf16, two boxes of 64 keys
    static constexpr int OFF_BAR = OFF_P + COLS * 256;
    static constexpr int OFF_MISC = OFF_BAR + 128;                     // tmem base, abort flag, status, bad rows of the tile before
    static constexpr int OFF_REF = OFF_MISC + 64;                      // [COLS] reference, base-2 units
    static constexpr int OFF_AT = OFF_REF + COLS * 4;                  // [2][COLS] position of the column's token, of two heads in turn
    static constexpr int OFF_ROW = OFF_AT + COLS * 8;                  // [2][COLS] its row among all (sequence, token, query head)
    static constexpr int OFF_ALPHA = OFF_ROW + COLS * 8;               // [COLS]
    static constexpr int OFF_WMAX = OFF_ALPHA + COLS * 4;              // [4 warps][COLS]
    static constexpr int TOTAL = OFF_WMAX + COLS * 16;
    static constexpr int DYN_BYTES = TOTAL + 1024;                     // slack for the 1024-byte alignment
};

// 8 values of every lane, each joined over the warp: lane l gets value l / 4.  The lanes halve the values that they hold three times, then
// join twice: 9 shuffles, where value by value takes 40.
template <typename F>
__device__ __forceinline__ float warp_of_8(const float* of, int lane, F join) {
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = of[x];
#pragma unroll
    for (int half = 4; half > 0; half >>= 1) {
        const bool upper = lane & (half * 4);
#pragma unroll
        for (int x = 0; x < half; ++x) {
            const float mine = upper ? v[x + half] : v[x], other = upper ? v[x] : v[x + half];
            v[x] = join(mine, __shfl_xor_sync(0xffffffffu, other, half * 4));
        }
    }
    v[0] = join(v[0], __shfl_xor_sync(0xffffffffu, v[0], 1));
    return join(v[0], __shfl_xor_sync(0xffffffffu, v[0], 2));
}
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
__global__ void __launch_bounds__(WinSmem<D, COLS, LOAD>::THREADS, WinSmem<D, COLS, LOAD>::CTAS)
decode_window_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ WindowParams p) {
    using SM = WinSmem<D, COLS, LOAD>;
    constexpr int ST = SM::STAGES;
    constexpr int BOX = 16384, NBOX = D / 64;
    constexpr int WORKERS = SM::WORKERS, THREADS = SM::THREADS, CONTROL = WORKERS / 32;        // CONTROL: the first control warp
    constexpr int WIDE = COLS / SM::HALVES;              // columns of a thread
    constexpr int CH = COLS <= 16 ? 8 : 16;              // of which it holds the scores at a time
    constexpr int QBOX = COLS * 128;                     // bytes of a 64-wide box of Q or P^T
    constexpr uint32_t IDESC_S = make_idesc(COLS, 0, 0), IDESC_O = make_idesc(COLS, 1, 0);
    constexpr bool PAGES = LOAD == WIN_PAGES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ long long s_scan[33], s_before;
    __shared__ int s_most, s_entry;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ps = p.page_size, G = p.G, E = p.S * p.groups;
    if (E > 32) {
        if (tid == 0) s_most = 0;
        __syncthreads();
    }
    pdl_wait();
    // ---- this CTA's share ----
    long long share, at, all, entry_before;
    int entry;
    // tiles of a CTA: not so few that a head is cut into more parts than there is room for: the first may be cut anywhere.
    // The second CTA of an SM starts 5 us after the first, which is worth two tiles: up to three tiles an SM are one CTA's (4 sequences of
    // 1000 to 2000 tokens, 392 tiles, 15.7 -> 14.0 us; 784 tiles would take 21.6 and not 20.2)
    auto share_of = [&](long long tiles, int most) {
        const long long even = max(max((tiles + gridDim.x - 1) / gridDim.x, ((long long)most + p.nsplit - 3) / (p.nsplit - 1)), 1ll);
        return tiles <= 3 * 148 ? max(even, (tiles + 147) / 148) : even;
    };
    auto head_of_workspace = [&]() {
        p.header[0] = (int32_t)WS_MAGIC;
        p.header[1] = KVS_OK;
        *reinterpret_cast<long long*>(p.header + WIN_SHARE_WORD) = share;
    };
    if (E <= 32) {
        // every warp for itself, a lane for an entry: no barrier of the CTA (calls that follow one another on the same caches: one windowed
        // sequence 9.9 -> 9.45 us, five drafted tokens of 24 sequences 92.7 -> 91.1, 16 of 500 to 6000 tokens the same)
        WindowUnit u;
        u.tiles = 0;
        if (lane < E) u.load(p, lane);
        long long upto = u.tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        all = __shfl_sync(0xffffffffu, upto, 31) * p.Hkv;
        share = share_of(all, __reduce_max_sync(0xffffffffu, u.tiles));
        at = share * blockIdx.x;
        const long long before = upto - u.tiles;
        if (blockIdx.x == 0 && warp == 0) {
            if (lane < E) p.entries[lane] = {before, u.tiles, 0};
            if (lane == 0) head_of_workspace();
        }
        if (at >= all) return;                             // the same in the whole CTA
        entry = __ffs(__ballot_sync(0xffffffffu, upto * p.Hkv > at)) - 1;
        entry_before = __shfl_sync(0xffffffffu, before, entry);
    } else {
        // every thread's first entry is kept: with no more entries than threads they are gone over once
        WindowUnit u;
        u.tiles = 0;
        if (tid < E) u.load(p, tid);
        long long rest = 0, first_sum;
        int most = u.tiles;
        for (int e = tid + THREADS; e < E; e += THREADS) {
            WindowUnit more;
            more.load(p, e);
            rest += more.tiles;
            most = max(most, more.tiles);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0 && most > 0) atomicMax(&s_most, most);
        const long long first_before = block_prefix((long long)u.tiles, s_scan, first_sum);
        all = first_sum;
        if (E > THREADS) {
            long long others;
            block_prefix(rest, s_scan, others);
            all += others;
        }
        all *= p.Hkv;
        share = share_of(all, s_most);
        at = share * blockIdx.x;
        if (blockIdx.x == 0 && tid == 0) head_of_workspace();
        if (at >= all && blockIdx.x != 0) return;          // the same in the whole CTA
        auto look = [&](int e, long long before) {         // is it this CTA's first entry; the first CTA writes all down
            if (e < E && blockIdx.x == 0) p.entries[e] = {before, u.tiles, 0};
            if (u.tiles > 0 && before * p.Hkv <= at && at < (before + u.tiles) * p.Hkv) {
                s_entry = e;
                s_before = before;
            }
        };
        look(tid, first_before);
        long long run = first_sum, here;
        for (int e0 = THREADS; e0 < E && (blockIdx.x == 0 || run * p.Hkv <= at); e0 += THREADS) {
            u.tiles = 0;
            if (e0 + tid < E) u.load(p, e0 + tid);
            const long long before = run + block_prefix((long long)u.tiles, s_scan, here);
            look(e0 + tid, before);
            run += here;
        }
        __syncthreads();
        if (at >= all) return;                             // the first CTA of a call without a tile
        entry = s_entry;
        entry_before = s_before;
    }
    const int my_tiles = (int)min(share, all - at);
    WindowCursor start;
    start.e = entry;
    start.before = entry_before;
    start.u.load(p, start.e);
    {
        const long long into = at - start.before * p.Hkv;
        start.g = (int)(into / start.u.tiles);
        start.i = (int)(into - (long long)start.g * start.u.tiles);
    }

    const uint32_t sraw = smem_u32(smem_raw), sbase = (sraw + 1023u) & ~1023u;
    uint8_t* sgen = smem_raw + (sbase - sraw);
    const uint32_t sK = sbase + SM::OFF_K, sV = sbase + SM::OFF_V, sQ = sbase + SM::OFF_Q, sP = sbase + SM::OFF_P, bars = sbase + SM::OFF_BAR;
    // K / V rows have landed; S^T is complete (one for each of its two buffers: the one of tile t + 2 waits for P^T of tile t, that of
    // t + 1 does not); P^T is written; the second product is complete (V and P^T consumed, O^T up to date); a head's queries are in place
    // K, V and the second products have one of each for every buffer; K of a buffer is consumed by S^T of its tile.
    const uint32_t bar_kfull = bars, bar_vfull = bars + 8 * ST, bar_kfree = bars + 16 * ST, bar_done = bars + 24 * ST, bar_s = bars + 32 * ST,
                   bar_p = bar_s + 16, bar_q = bar_s + 24;
    // a buffer's barrier and its phase at tile `it`
    auto stage_of = [](int it) { return (uint32_t)(it % ST); };
    auto phase_of = [](int it) { return (uint32_t)(it / ST & 1); };
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
        for (int b = 0; b < ST; ++b) {
            mbar_init(bar_kfull + 8 * b, SM::K_WARPS);
            mbar_init(bar_vfull + 8 * b, PAGES ? 2 : 32 * SM::V_WARPS);
            mbar_init(bar_kfree + 8 * b, 1);
            mbar_init(bar_done + 8 * b, 1);
        }
        mbar_init(bar_s, 1);
        mbar_init(bar_s + 8, 1);
        mbar_init(bar_p, WORKERS);
        mbar_init(bar_q, WORKERS);
        fence_mbar_init();
    }
    if (warp == CONTROL) {
        tmem_alloc(smem_u32(s_tmem), 4 * COLS);            // S^T twice and O^T, in a power of two
        tmem_relinquish();
    } else if (tid < COLS) {
        s_ref[tid] = WIN_AHEAD;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_S = *s_tmem, tmem_O = tmem_S + 2 * COLS;
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

    if (warp >= CONTROL) {
        // ================= control warps: one issues the products, the others load K and V =================
        reg_dec<SM::CONTROL_REGS>();
        const bool leader = elect_one();
        const int ppt = PAGES ? 128 / ps : 0;                  // pages per tile
        WindowCursor c = start;
        if (warp == CONTROL) {
            const uint64_t dK = smem_desc(sK, 16, 1024), dQ = smem_desc(sQ, 16, 1024);
            const uint64_t dV = smem_desc(sV, D == 128 ? BOX : 0, 1024), dP = smem_desc(sP, 16, 1024);
            int heads = 0;
            auto scores = [&](int it, bool head) {             // S^T of tile `it`; the first of a head waits for its queries
                if (head) mbar_wait(bar_q, heads++ & 1, abort_flag, status);
                mbar_wait(bar_kfull + 8 * stage_of(it), phase_of(it), abort_flag, status);
                tc_fence_after();
                const uint64_t dKt = dK + (uint64_t)(stage_of(it) * (SM::TILE_BYTES >> 4));
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {          // S^T = K Q^T, 16 elements of d per step
                    const uint64_t offk = (uint64_t)(((kk >> 2) * BOX + (kk & 3) * 32) >> 4);
                    const uint64_t offq = (uint64_t)(((kk >> 2) * QBOX + (kk & 3) * 32) >> 4);
                    if (leader) mma_ss(tmem_S + (it & 1) * COLS, dKt + offk, dQ + offq, IDESC_S, kk > 0);
                }
                if (leader) {
                    mma_commit(bar_s + (it & 1) * 8);
                    mma_commit(bar_kfree + 8 * stage_of(it));
                }
            };
            scores(0, true);
            bool first = true;
            for (int it = 0; it < my_tiles; ++it) {
                // the next tile's scores while this one's are in work; those of another head behind P^T, as their queries come behind it
                const bool more = it + 1 < my_tiles;
                if (more) c.next(p);
                const bool head = c.i == 0;
                if (more && !head) scores(it + 1, false);
                mbar_wait(bar_p, it & 1, abort_flag, status);
                mbar_wait(bar_vfull + 8 * stage_of(it), phase_of(it), abort_flag, status);
                tc_fence_after();
                const uint64_t dVt = dV + (uint64_t)(stage_of(it) * (SM::TILE_BYTES >> 4));
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {               // O^T += V^T P^T, 16 keys per step
                    const uint64_t offp = (uint64_t)(((kk >> 2) * QBOX + (kk & 3) * 32) >> 4);
                    if (leader) mma_ss(tmem_O, dVt + (uint64_t)(kk * 128), dP + offp, IDESC_O, !first || (kk > 0));
                }
                if (leader) mma_commit(bar_done + 8 * stage_of(it));
                first = head;
                if (more && head) scores(it + 1, true);
            }
        } else if (PAGES || warp <= CONTROL + SM::K_WARPS) {
            // TMA.  PAGES: lane i has page i of the tile, if some query sees a row of it (of V every second page is the other warp's).
            // ROWS: K alone, lane L has the rows 4 L .. 4 L + 3 (rows past the end repeat the last one: their scores are masked), if some
            // query sees one of them, and if they are this warp's.  The block-table entries are read a tile ahead.
            const bool k_rows = !PAGES || warp == CONTROL + 1;
            const CUtensorMap* map = k_rows ? &tm_k : &tm_v;
            const uint32_t base = k_rows ? sK : sV, fulls = k_rows ? bar_kfull : bar_vfull, frees = k_rows ? bar_kfree : bar_done;
            const bool mine = PAGES ? lane < ppt && (k_rows || (lane & 1) == (warp - CONTROL - 2)) : lane % SM::K_WARPS == warp - CONTROL - 1;
            int id[PAGES ? 1 : 4], off[PAGES ? 1 : 4], g = 0;
            bool need = false;
            auto fetch = [&]() {                               // of the tile at the cursor
                const int32_t* bt = p.block_table + (size_t)c.u.s * p.max_pages;
                const int k0 = c.u.key_of(c.i), a = k0 + lane * (PAGES ? ps : 4), e = min(a + (PAGES ? ps : 4), c.u.end);
                need = mine && a < e && (a < c.u.head || e > c.u.lo);
                g = c.g;
                if constexpr (PAGES) {
                    if (need) id[0] = bt[(k0 >> 7) * ppt + lane];
                } else if (need) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int en;
                        split_token(min(a + j, c.u.end - 1), en, off[j]);
                        id[j] = bt[en];
                    }
                }
            };
            fetch();
            for (int it = 0; it < my_tiles; ++it) {
                const uint32_t dst = base + stage_of(it) * SM::TILE_BYTES, full = fulls + 8 * stage_of(it);
                if (it >= ST) mbar_wait(frees + 8 * stage_of(it), phase_of(it - ST), abort_flag, status);       // the buffer's last tile is consumed
                const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, need));
                if (leader) mbar_expect_tx(full, boxes * (uint32_t)((PAGES ? ps : 4) * D * 2));
                __syncwarp();
                if (need) {
                    if constexpr (PAGES) {
                        const int row = checked_page(id[0]) * ps;
#pragma unroll
                        for (int b = 0; b < NBOX; ++b) tma_load_3d(dst + b * BOX + (uint32_t)(lane * ps) * 128u, map, b * 64, g, row, full);
                    } else {
                        int row[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) row[j] = checked_page(id[j]) * ps + off[j];
#pragma unroll
                        for (int b = 0; b < NBOX; ++b)
                            tma_gather4(dst + b * BOX + (uint32_t)lane * 512u, map, g * D + b * 64, row[0], row[1], row[2], row[3], full);
                    }
                }
                __syncwarp();
                if (it + 1 < my_tiles) {
                    c.next(p);
                    fetch();
                }
            }
        } else {
            // V by rows: 16 bytes of a row a lane, LPR lanes a row; rows that no query sees are filled with zeros.  A lane has the block-table
            // entries of IDS of its warp's rows, read a tile ahead, and hands their rows of the cache to the lanes that copy.
            constexpr int LPR = D / 8, RPW = 32 / LPR, ROWS = 128 / SM::V_WARPS, IDS = ROWS / 32, NIT = ROWS / RPW;
            const int part = warp - CONTROL - 1 - SM::K_WARPS, l = lane % LPR;
            auto row_of = [&](int i) { return i / RPW * (SM::V_WARPS * RPW) + part * RPW + i % RPW; };         // the warp's i-th row in the tile
            int id[IDS];
            auto fetch = [&]() {
                const int32_t* bt = p.block_table + (size_t)c.u.s * p.max_pages;
#pragma unroll
                for (int h = 0; h < IDS; ++h) {
                    int en, o;
                    split_token(min(c.u.key_of(c.i) + row_of(lane + 32 * h), c.u.end - 1), en, o);
                    id[h] = bt[en];
                }
            };
            fetch();
            for (int it = 0; it < my_tiles; ++it) {
                if (it >= ST) mbar_wait(bar_done + 8 * stage_of(it), phase_of(it - ST), abort_flag, status);
                const int k0 = c.u.key_of(c.i);
                int row[IDS];                                    // of the cache; -1: seen by no query
#pragma unroll
                for (int h = 0; h < IDS; ++h) {
                    const int k = k0 + row_of(lane + 32 * h);
                    int en, o;
                    split_token(min(k, c.u.end - 1), en, o);
                    const int page = checked_page(id[h]);
                    row[h] = c.u.seen_by_some(k) ? page * ps + o : -1;
                }
                const __nv_bfloat16* src = p.v_cache + (size_t)c.g * D + l * 8;
#pragma unroll
                for (int j = 0; j < NIT; ++j) {
                    const int i = j * RPW + lane / LPR, r = row_of(i), from = __shfl_sync(0xffffffffu, row[j * RPW / 32], i & 31);
                    const uint32_t dst = (uint32_t)((l >> 3) * BOX + r * 128 + (((l & 7) ^ (r & 7)) << 4)), bytes = from >= 0 ? 16u : 0u;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sV + stage_of(it) * SM::TILE_BYTES + dst), "l"(src + (size_t)max(from, 0) * p.Hkv * D), "r"(bytes)
                                 : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (it + 1 < my_tiles) {
                    c.next(p);
                    fetch();
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                fence_proxy_async();                           // the tensor core reads them
                mbar_arrive(bar_vfull + 8 * stage_of(it));
            }
        }
    } else {
        // ================= softmax warps =================
        reg_inc<SM::WORKER_REGS>();
        const int key = tid & 127, col0 = tid < 128 ? 0 : WIDE;          // this thread's key of a tile (and column d of O^T), its first column
        const uint32_t lane_sel = (uint32_t)((warp & 3) * 32) << 16;
        WindowCursor c = start;
        float l_part[WIDE];
#pragma unroll
        for (int i = 0; i < WIDE; ++i) l_part[i] = 0.f;
        auto sees = [&](int j, int at) { return j <= at && (j < p.sinks || at - j < p.window); };
        // O^T += weight x V for the rows of the tile at k0 that were kept out of the second product.  O^T is up to date, P^T still there.
        const int* at_of = s_at;              // of the columns of the head in work
        auto patch = [&](int k0) {
            const int32_t* bt = p.block_table + (size_t)c.u.s * p.max_pages;
            const int cols = c.u.cols;
            for (int r0 = 0; r0 < 128; r0 += 32)
                for (uint32_t m = s_bad[r0 >> 5]; m; m &= m - 1) {
                    const int r = r0 + __ffs(m) - 1;
                    int en, o;
                    split_token(k0 + r, en, o);
                    const size_t row = (size_t)checked_page(bt[en]) * ps + o;
                    const float v = __bfloat162float(p.v_cache[(row * p.Hkv + c.g) * D + key % D]);
                    for (int c0 = col0; c0 < min(cols, col0 + WIDE); c0 += 16) {
                        uint32_t x[16];
                        tmem_ld16(tmem_O + c0 + lane_sel, x);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (sees(k0 + r, at_of[c0 + i])) {
                                const uint8_t* w = sgen + SM::OFF_P + (r >> 6) * QBOX + (c0 + i) * 128 + ((((r & 63) >> 3) ^ (i & 7)) << 4) + ((r & 7) << 1);
                                x[i] = __float_as_uint(__uint_as_float(x[i]) + __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(w)) * v);
                            }
                        tmem_st16(tmem_O + c0 + lane_sel, x);
                        tmem_wait_st();
                    }
                }
        };
        // the queries of the head at the cursor, columns' positions and rows in half `which`
        auto load_q = [&](int which) {
            if (tid < COLS) {
                const int t = tid / G;
                s_at[which * COLS + tid] = tid < c.u.cols ? c.u.at0 + t : -1;
                s_row[which * COLS + tid] = tid < c.u.cols ? (c.u.s * p.n_new + c.u.tok0 + t) * p.Hq + c.g * G + (tid - t * G) : -1;
            }
            named_bar_sync(1, WORKERS);
            // column, 16-byte chunk of its row: box, then chunk ^ (column % 8) of the 128-byte row; columns past the last are zero
            constexpr int NQ = COLS * (D / 8) / WORKERS;     // chunks a thread, all on their way before the first is stored
            uint4 v[NQ];
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const int i = tid + k * WORKERS, row = s_row[which * COLS + i / (D / 8)];
                v[k] = row >= 0 ? *reinterpret_cast<const uint4*>(p.q + (size_t)row * D + (i % (D / 8)) * 8) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const int i = tid + k * WORKERS, col = i / (D / 8), c16 = i % (D / 8);
                *reinterpret_cast<uint4*>(sgen + SM::OFF_Q + (c16 >> 3) * QBOX + col * 128 + (((c16 & 7) ^ (col & 7)) << 4)) = v[k];
            }
            fence_proxy_async();
            mbar_arrive(bar_q);
        };
        load_q(0);
        bool to_patch = false;
        int before_k0 = 0, left = my_tiles, which = 0;
        bool first = true;                                      // of the head's tiles in this CTA
        for (int it = 0; it < my_tiles; ++it) {
            const WindowUnit& u = c.u;
            const int k0 = u.key_of(c.i), j = k0 + key, cols = u.cols, at0 = u.at0, end = u.end;
            at_of = s_at + which * COLS;
            const bool last = --left == 0 || c.i + 1 == u.tiles;
            mbar_wait(bar_s + (it & 1) * 8, (it >> 1) & 1, abort_flag, status);          // S^T ready
            tc_fence_after();
            // some query does not see some key of the tile
            const bool masked = k0 + 127 > at0 || !(k0 + 127 < p.sinks || end - 1 - k0 < p.window);
            // scores of CH columns from c0, read where they are needed: there is no room to hold them all.  Columns come in blocks without a
            // branch inside, so that a block's loads and exponentials overlap.
            auto scores = [&](int c0, float (&sc)[CH], float (&ref)[CH]) {
                uint32_t r[16];
                tmem_ld16(tmem_S + (it & 1) * COLS + c0 + lane_sel, r);
#pragma unroll
                for (int x = 0; x < CH; x += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(s_ref + c0 + x);
                    ref[x] = y.x;
                    ref[x + 1] = y.y;
                    ref[x + 2] = y.z;
                    ref[x + 3] = y.w;
                }
                tmem_wait_ld();
#pragma unroll
                for (int x = 0; x < CH; ++x) sc[x] = __uint_as_float(r[x]) * p.scale_log2;
                if (masked) {
#pragma unroll
                    for (int x = 0; x < CH; ++x) sc[x] = sees(j, at_of[c0 + x]) ? sc[x] : -INFINITY;
                }
            };
            bool above = false;
#pragma unroll
            for (int c0 = 0; c0 < WIDE; c0 += CH)
                if (col0 + c0 < cols) {
                    float sc[CH], ref[CH];
                    scores(col0 + c0, sc, ref);
#pragma unroll
                    for (int x = 0; x < CH; ++x) above |= first ? !(fabsf(sc[x]) <= WIN_AHEAD + WIN_OVER) : sc[x] - ref[x] > WIN_OVER;
                }
            // the same decision in every thread.  In a head's first tile every column has to have seen a key: masked ones are looked at
            const bool grow = group_any(1, WORKERS, above || (first && masked));
            if (it > 0) {                                       // P^T is free, O^T up to date
                mbar_wait(bar_done + 8 * stage_of(it - 1), phase_of(it - 1), abort_flag, status);
                tc_fence_after();
            }
            if (to_patch) {                                     // the same decision in every thread
                patch(before_k0);
                named_bar_sync(1, WORKERS);                     // P^T is written again below
            }
            if (grow) {
                // the columns' maxima over the tile; the references that are too low move there
#pragma unroll
                for (int c0 = 0; c0 < WIDE; c0 += CH)
                    if (col0 + c0 < cols) {
                        float sc[CH], ref[CH];
                        scores(col0 + c0, sc, ref);
#pragma unroll
                        for (int b = 0; b < CH; b += 8) {
                            const float m = warp_of_8(sc + b, lane, [](float x, float y) { return fmaxf(x, y); });
                            if ((lane & 3) == 0) s_wmax[(warp & 3) * COLS + col0 + c0 + b + (lane >> 2)] = m;
                        }
                    }
                named_bar_sync(1, WORKERS);
                if (tid < COLS) {
                    const float top = fmaxf(fmaxf(s_wmax[tid], s_wmax[COLS + tid]), fmaxf(s_wmax[2 * COLS + tid], s_wmax[3 * COLS + tid]));
                    const float ref = s_ref[tid];
                    float to = ref;
                    if (tid < cols) to = first ? (top > -INFINITY ? top + WIN_AHEAD : WIN_UNSET) : top - ref > WIN_OVER ? top + WIN_AHEAD : ref;
                    s_alpha[tid] = first ? 1.f : fast_exp2(ref - to);        // nothing has been added up before the first
                    s_ref[tid] = to;
                }
                named_bar_sync(1, WORKERS);
#pragma unroll
                for (int x = 0; x < WIDE; ++x) l_part[x] *= s_alpha[col0 + x];
                if (!first) {                     // O^T row d = key
                    for (int c0 = col0; c0 < min(cols, col0 + WIDE); c0 += 16) {
                        uint32_t o[16];
                        tmem_ld16(tmem_O + c0 + lane_sel, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * s_alpha[c0 + x]);
                        tmem_st16(tmem_O + c0 + lane_sel, o);
                        tmem_wait_st();
                    }
                }
            }
            // weights of this key -> P^T[column][key] (bf16), row `column` of box key / 64
            uint8_t* prow = sgen + SM::OFF_P + (key >> 6) * QBOX + ((key & 7) << 1);
            const int chunk = (key & 63) >> 3;
#pragma unroll
            for (int c0 = 0; c0 < WIDE; c0 += CH)
                if (col0 + c0 < cols) {
                    float sc[CH], ref[CH];
                    scores(col0 + c0, sc, ref);
#pragma unroll
                    for (int x = 0; x < CH; ++x) {
                        const float w = fast_exp2(sc[x] - ref[x]);
                        l_part[c0 + x] += w;
                        *reinterpret_cast<__nv_bfloat16*>(prow + (col0 + c0 + x) * 128 + ((chunk ^ (x & 7)) << 4)) = __float2bfloat16(w);
                    }
                }
            to_patch = false;
            if (masked) {                         // the same decision in every thread
                mbar_wait(bar_vfull + 8 * stage_of(it), phase_of(it), abort_flag, status);
                bool clear = tid < 128 && !u.seen_by_some(j), bad = false;
                uint4* vrow = reinterpret_cast<uint4*>(sgen + SM::OFF_V + stage_of(it) * SM::TILE_BYTES + key * 128);
                if (tid < 128 && !clear && !(sees(j, at0) && sees(j, end - 1))) {
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
                if (lane == 0 && warp < 4) s_bad[warp] = bads;
                if (clear || bad) {
#pragma unroll
                    for (int b = 0; b < NBOX; ++b)
#pragma unroll
                        for (int i = 0; i < 8; ++i) vrow[b * (BOX / 16) + i] = make_uint4(0, 0, 0, 0);
                }
                to_patch = group_any(1, WORKERS, bad);
            }
            fence_proxy_async();      // P^T and the V rows written by this thread visible to the tensor core's reads of shared memory
            tc_fence_before();
            mbar_arrive(bar_p);
            first = last;
            if (!last) {
                before_k0 = k0;
                ++c.i;
                continue;
            }
            // ---- the head's part is done.  Its result's place first, then the next head's queries (K is there already) ----
            const int part = (int)(blockIdx.x - (c.before * p.Hkv + (long long)c.g * u.tiles) / share);
            const int result = which * COLS;
            const WindowCursor done = c;
            if (left > 0) {
                c.next_unit(p);
                which ^= 1;
                load_q(which);
            }
            mbar_wait(bar_done + 8 * stage_of(it), phase_of(it), abort_flag, status);
            tc_fence_after();
            if (to_patch) {
                const WindowCursor next = c;
                c = done;
                patch(k0);
                c = next;
                to_patch = false;
            }
#pragma unroll
            for (int c0 = 0; c0 < WIDE; c0 += 8)
                if (col0 + c0 < cols) {
                    const float sum = warp_of_8(l_part + c0, lane, [](float x, float y) { return x + y; });
                    if ((lane & 3) == 0) s_wmax[(warp & 3) * COLS + col0 + c0 + (lane >> 2)] = sum;
                }
            for (int c0 = col0; c0 < min(cols, col0 + WIDE); c0 += 16) {
                uint32_t o[16];
                tmem_ld16(tmem_O + c0 + lane_sel, o);
                tmem_wait_ld();
                if (key < D) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const int row = s_row[result + c0 + x];
                        if (row >= 0) p.part_o[((size_t)row * p.nsplit + part) * D + key] = __uint_as_float(o[x]);
                    }
                }
            }
            named_bar_sync(1, WORKERS);
            if (tid < cols) {
                const float ref = s_ref[tid];
                float* ml = p.part_ml + ((size_t)s_row[result + tid] * p.nsplit + part) * 2;
                ml[0] = ref == WIN_UNSET ? -INFINITY : ref;
                ml[1] = flagged_sum(s_wmax[tid] + s_wmax[COLS + tid] + s_wmax[2 * COLS + tid] + s_wmax[3 * COLS + tid], *(volatile int32_t*)status);
            }
            if (left > 0) {
                if (tid < COLS) s_ref[tid] = WIN_AHEAD;
#pragma unroll
                for (int x = 0; x < WIDE; ++x) l_part[x] = 0.f;
                named_bar_sync(1, WORKERS);                         // the references are read by all
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == CONTROL) {
        __syncwarp();
        tmem_dealloc(tmem_S, 4 * COLS);
    }
}

// A warp for a row (sequence, token, query head): its head's tiles were `count` CTAs' work.  Loads of 8 parts at a time and three CTAs an SM
// (16 and two: 24 sequences with 5 new tokens of 28 heads 95.6 -> 93.3 us, a round of 16 with 32 heads 62.1 -> 59.9).
template <int D, int PART>
__global__ void __launch_bounds__(32 * MERGE_WARPS, 3) window_merge_kernel(MergeParams m, const WindowEntry* entries, int Hq, int G, int Hkv, int n_new, int groups,
                                                          int group_tokens) {
    pdl_wait();
    const unsigned at_row = merge_row();
    if (at_row >= (unsigned)m.rows) return;
    const int row = (int)at_row;
    const int token = row / Hq, g = (row - token * Hq) / G, s = token / n_new;
    const WindowEntry e = entries[s * groups + (token - s * n_new) / group_tokens];
    const long long share = *reinterpret_cast<const long long*>(m.header + WIN_SHARE_WORD), at = e.before * Hkv + (long long)g * e.tiles;
    const int count = e.tiles == 0 ? 0 : (int)((at + e.tiles - 1) / share - at / share + 1);
    decode_merge_row<D, PART>(m, row, threadIdx.x & 31, count);
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

template <int D, int COLS, int LOAD>
int launch_window(const CUtensorMap& tk, const CUtensorMap& tv, const WindowParams& p, long long most_tiles, cudaStream_t st) {
    using SM = WinSmem<D, COLS, LOAD>;
    auto kern = decode_window_kernel<D, COLS, LOAD>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::DYN_BYTES) != cudaSuccess) return cuda_refused();
    const long long ctas = most_tiles < 148 * SM::RESIDENT ? most_tiles : 148 * SM::RESIDENT;        // one wave
    return launch_after(kern, dim3((unsigned)(ctas < 1 ? 1 : ctas)), SM::THREADS, SM::DYN_BYTES, st, tk, tv, p);
}
template <int D, int COLS>
int launch_window(const CUtensorMap& tk, const CUtensorMap& tv, const WindowParams& p, long long most_tiles, bool pages, cudaStream_t st) {
    return pages ? launch_window<D, COLS, WIN_PAGES>(tk, tv, p, most_tiles, st) : launch_window<D, COLS, WIN_ROWS>(tk, tv, p, most_tiles, st);
}
template <int D>
int launch_window_cols(const CUtensorMap& tk, const CUtensorMap& tv, const WindowParams& p, const MergeParams& m, long long most_tiles, bool pages,
                       cudaStream_t st) {
    const int cols = p.G * p.group_tokens;
    const int rc = cols <= 16 ? launch_window<D, 16>(tk, tv, p, most_tiles, pages, st)
                 : cols <= 32 ? launch_window<D, 32>(tk, tv, p, most_tiles, pages, st)
                              : launch_window<D, 64>(tk, tv, p, most_tiles, pages, st);
    if (rc != KVS_OK) return rc;
    return launch_after(p.nsplit <= 4 ? window_merge_kernel<D, 4> : window_merge_kernel<D, 8>, merge_ctas(m.rows), 32 * MERGE_WARPS, 0, st, m, p.entries, p.Hq,
                        p.G, p.Hkv, p.n_new, p.groups, p.group_tokens);
}
// rows' results, room for one part more than num_splits (a border may fall anywhere in a head's tiles); then the entries
size_t window_entries_offset(int num_seqs, int n_new, int Hq, int head_dim, int num_splits) {
    return DEC_WS_HEADER + align_up(sizeof(float) * (size_t)num_seqs * n_new * Hq * ((size_t)num_splits + 1) * (head_dim + 2), 256);
}
}  // namespace

extern "C" int kvs_decode_window_num_splits(int num_seqs, int n_new, int Hq, int Hkv, int max_tokens, int window, int sinks) {
    if (num_seqs <= 0 || n_new <= 0 || Hq <= 0 || Hkv <= 0 || max_tokens <= 0 || window <= 0 || sinks < 0) return 1;
    if (Hq % Hkv != 0 || Hq / Hkv > WIN_MOST_COLS) return 1;
    // every CTA of a wave of three an SM has an equal share; a sequence four times as long as the mean is still cut as small as that
    const long long units = (long long)num_seqs * window_groups(Hq / Hkv, n_new) * Hkv, tiles = window_tiles(n_new, max_tokens, window, sinks);
    long long n = (4 * 3 * 148 + units - 1) / units;
    if (n > tiles) n = tiles;
    return (int)(n > 64 ? 64 : n < 1 ? 1 : n);
}

extern "C" size_t kvs_decode_window_workspace_bytes(int num_seqs, int n_new, int Hq, int Hkv, int head_dim, int num_splits) {
    if (num_seqs < 0 || n_new < 0 || Hq <= 0 || Hkv <= 0 || head_dim <= 0 || num_splits <= 0) return 0;
    if (Hq % Hkv != 0 || Hq / Hkv > WIN_MOST_COLS) return 0;
    return window_entries_offset(num_seqs, n_new, Hq, head_dim, num_splits) + sizeof(WindowEntry) * (size_t)num_seqs * window_groups(Hq / Hkv, n_new);
}

extern "C" int kvs_decode_attn_window(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* n_tokens,
                                      int num_seqs, int n_new, int Hq, int Hkv, int head_dim, int page_size, int max_pages, int num_pages, float softmax_scale,
                                      int window, int sinks, int num_splits, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                      kvs_stream_t stream) {
    if (num_seqs < 0 || n_new < 0 || Hq <= 0 || Hkv <= 0 || page_size <= 0 || max_pages <= 0 || num_pages <= 0 || num_splits <= 0 || window <= 0 || sinks < 0)
        return KVS_ERR_INVALID_ARG;
    if (softmax_scale < 0.f || softmax_scale != softmax_scale) return KVS_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return KVS_ERR_UNSUPPORTED;
    if (Hq % Hkv != 0 || Hq / Hkv > WIN_MOST_COLS) return KVS_ERR_UNSUPPORTED;
    if (num_seqs == 0 || n_new == 0) return KVS_OK;
    const int G = Hq / Hkv, groups = window_groups(G, n_new);
    if ((long long)num_seqs * groups > 0x7fffffffLL || (long long)num_seqs * n_new * Hq > 0x7fffffffLL) return KVS_ERR_UNSUPPORTED;
    if ((long long)num_pages * page_size > 0x7fffffffLL || (long long)max_pages * page_size > 0x7fffff00LL || (long long)Hkv * head_dim > 0x7fffffffLL)
        return KVS_ERR_UNSUPPORTED;
    if (!q || !k_cache || !v_cache || !block_table || !n_tokens || !out || !lse || !workspace) return KVS_ERR_INVALID_ARG;
    if ((((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15) != 0 || ((uintptr_t)workspace & 255) != 0 ||
        (((uintptr_t)block_table | (uintptr_t)n_tokens | (uintptr_t)lse) & 3) != 0)
        return KVS_ERR_ALIGNMENT;
    if (workspace_bytes < kvs_decode_window_workspace_bytes(num_seqs, n_new, Hq, Hkv, head_dim, num_splits)) return KVS_ERR_WORKSPACE;
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
    p.nsplit = num_splits + 1;
    p.groups = groups;
    p.group_tokens = (n_new + groups - 1) / groups;
    p.window = window;
    p.sinks = sinks;
    p.header = (int32_t*)workspace;
    p.scale_log2 = (softmax_scale == 0.f ? 1.0f / sqrtf((float)head_dim) : softmax_scale) * 1.4426950408889634f;
    p.part_o = (float*)((char*)workspace + DEC_WS_HEADER);
    p.part_ml = p.part_o + (size_t)num_seqs * n_new * Hq * p.nsplit * head_dim;
    p.entries = (WindowEntry*)((char*)workspace + window_entries_offset(num_seqs, n_new, Hq, head_dim, num_splits));
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
    const MergeParams m = {p.part_o, p.part_ml, (__nv_bfloat16*)out, lse, p.header, num_seqs * n_new * Hq, p.nsplit};
    const long long most_tiles = window_tiles(n_new, max_pages * page_size, window, sinks) * num_seqs * groups * Hkv;
    return head_dim == 64 ? launch_window_cols<64>(tk, tv, p, m, most_tiles, pages, st) : launch_window_cols<128>(tk, tv, p, m, most_tiles, pages, st);
}
