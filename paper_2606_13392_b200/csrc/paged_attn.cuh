// Softmax attention of new tokens over a paged cache (include/msa.h: msa_paged_attn):
//   out[t, h] = sum_{j <= pos(t)} softmax_j(scale <q[t, h], k_j>) v_j,   lse = log sum_j exp(scale <q, k_j>)
//
// Unit of work: 128 keys against one tile of query rows of a (sequence, KV head).  A row is a (token, head of the
// group) pair, so the G heads of a group share every K/V tile: a context holds TPT = 128 / G tokens.  Sequences of
// more new tokens than that give a CTA two contexts of consecutive tokens that share the K/V tiles (256 rows per
// 64 KB); short ones (decode) put both contexts on the same rows, taking key tiles in turn, and merge at the end.
//
// The units of all tiles form one line (sequence, head, tile, key tile) and every CTA takes an equal stretch of it:
// ragged batches balance whatever their lengths.  Beginning and ending a tile takes about as long as kPagedTileCost units,
// which stand on the line behind the tile's own.  A tile that a stretch boundary cuts leaves fp32
// partials (at most two per CTA), merged by paged_combine_kernel; all others are written directly.
//
// Measured (64 query, 8 KV heads): 4096 new tokens on 28K in 3.8 - 4.6 ms, 0.9 - 1.08 PFLOP/s at the board's power limit,
// 57 % of the tensor pipe's cycles and 58 % of the exponential unit's; one token each of 64 sequences of up to 32K in 590 -
// 680 us, 90 - 104 % of the copy bandwidth; 2 - 7 tokens each of 16 sequences in 86 - 92 us, 74 - 78 %; one token on 2K in 16
// us.  On fp8 caches: 4096 on 28K in 3.7 - 3.8 ms, 512 on 7K in 153 us (0.8 PFLOP/s), 2 - 7 tokens each of 16 sequences in
// 102 us (33 % of the copy bandwidth: tiles are read, widened and written back in shared memory).
#pragma once

#include "norm_rope.cuh"
#include "tc_common.cuh"

namespace msa {

constexpr int kPagedKeys = 128;   // keys of a tile
constexpr int kPagedKStages = 2, kPagedVStages = 3;  // (V waits for the softmax, K does not)
constexpr int kPagedSlotRows = 256;                  // rows of a partial: two contexts

struct PagedAttnArgs {
    PagedView c;
    int G, TPT;          // query heads per KV head; tokens per context
    int tile_tokens;     // tokens of a query tile of a sequence with more than TPT: two contexts, or one
    int slot_rows;       // rows of a partial
    int n_tokens;
    int min_len, max_len;  // new tokens of the sequences that this launch takes (another takes the rest)
    float scale_log2e;
    __nv_bfloat16* out;  // [n_tokens, H_kv*G, 128]
    float* lse;          // [n_tokens, H_kv*G] or null
    // partials: CTA i owns slots 2i (a tile begun by an earlier CTA) and 2i+1 (a tile that a later one ends)
    float* part_o;       // [slot][slot_rows][128], not normalised
    float2* part_ml;     // [slot][slot_rows] reference maximum (log2 units) and sum
    int4* ends;          // [CTA][2]: see PagedEnds
};

// What paged_combine_kernel has to know about a CTA.
//   first: 0 no work; 1 its first tile came from an earlier CTA and goes on in a later one; 2 came from an earlier
//          one and ends here; 3 begins here
//   open:  its last tile begins here and ends in a later CTA; q_row, tokens, head describe it
struct PagedEnds { int first, open, q_row, tokens, head, pad[3]; };
static_assert(sizeof(PagedEnds) == 32, "two int4");

// ---------------------------------------------------------------- the line of units
struct PagedSeq { int q_row, q_len, kv, base, tile_tokens, n_tiles; };

__host__ __device__ __forceinline__ int64_t paged_cap(const PagedView& c) { return (int64_t)c.max_pages * c.page_size; }

__host__ __device__ __forceinline__ PagedSeq paged_seq(const PagedAttnArgs& a, int s) {
    PagedSeq q;
    const int lo = max(a.c.cu_q[s], 0), end = a.c.cu_q[s + 1], hi = min(end, a.n_tokens);  // (rows that are not there: none)
    q.q_row = lo;
    q.q_len = max(hi - lo, 0);
    if (q.q_len < a.min_len || q.q_len > a.max_len) q.q_len = 0;  // (another launch's: no rows here)
    q.kv = (int)min((int64_t)max(a.c.kv_lens[s], 0), paged_cap(a.c));
    q.base = q.kv - max(end - lo, 0);  // position of the first new token
    q.tile_tokens = q.q_len <= a.TPT ? a.TPT : a.tile_tokens;
    q.n_tiles = (q.q_len + q.tile_tokens - 1) / q.tile_tokens;
    return q;
}

// Key tiles of query tile t: up to its last token's position (at least one: a tile of rows that see nothing is
// visited too, to write their zeros).
__host__ __device__ __forceinline__ int paged_blocks(const PagedSeq& q, int t) {
    const int64_t last = (int64_t)max(q.base, 0) + min((int64_t)(t + 1) * q.tile_tokens, (int64_t)q.q_len);
    return (int)((last + kPagedKeys - 1) / kPagedKeys);
}

// sum over i < n of floor((a i + b) / m), a, b >= 0: Euclid's steps on (a, m).  T: 32 bits where a n + b fits (they
// divide several times faster, and a CTA's prologue takes some twenty of these sums).
template <class T>
__host__ __device__ inline int64_t floor_sum_of(T n, T m, T a, T b) {
    int64_t sum = 0;
    while (n > 0) {
        const T qa = a / m, qb = b / m;
        sum += (int64_t)n * ((int64_t)n - 1) / 2 * (int64_t)qa + (int64_t)n * (int64_t)qb;
        a -= qa * m;
        b -= qb * m;
        const T y = a * n + b;
        n = y / m;
        b = y - n * m;
        const T t = m;
        m = a;
        a = t;
        if (m == 0) break;
    }
    return sum;
}
__host__ __device__ inline int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
    if (a * n + b < (1ll << 31)) return floor_sum_of<uint32_t>((uint32_t)n, (uint32_t)m, (uint32_t)a, (uint32_t)b);
    return floor_sum_of<int64_t>(n, m, a, b);
}

// (64 sequences of one token on up to 1000: 75 us without, 63, 58, 61 us with 2, 3, 5; 4096 tokens on themselves 370, 306,
// 301, 303 us)
constexpr int kPagedTileCost = 3;

// Units of the first t query tiles of one head, their cost included.
__host__ __device__ inline int64_t paged_units_before(const PagedSeq& q, int t) {
    if (t <= 0) return 0;
    const int full = min(t, q.n_tiles - 1);  // (the last tile may be short)
    int64_t u = floor_sum(full, kPagedKeys, q.tile_tokens, (int64_t)max(q.base, 0) + q.tile_tokens + kPagedKeys - 1);
    if (t >= q.n_tiles) u += paged_blocks(q, q.n_tiles - 1);
    return u + (int64_t)min(t, q.n_tiles) * kPagedTileCost;
}

// Units of a sequence.
__host__ __device__ inline int64_t paged_units(const PagedAttnArgs& a, const PagedSeq& q) {
    if (q.n_tiles <= 1) return q.n_tiles == 0 ? 0 : (int64_t)a.c.H_kv * (paged_blocks(q, 0) + kPagedTileCost);
    return (int64_t)a.c.H_kv * paged_units_before(q, q.n_tiles);
}

// A place on the line; seq = batch: its end.
struct PagedPlace { int seq, head, tile, blk; };

// Unit `u` of sequence s.  blk = nb: the tile's end.  snap: places inside long tiles move to the nearest eighth of the tile, so that CTAs that
// read the same long K/V do it in step (see launch_paged_attn).
__host__ __device__ inline PagedPlace paged_place(const PagedAttnArgs& a, int s, int64_t u, int64_t snap_keys) {
    const PagedSeq q = paged_seq(a, s);
    const int64_t per_head = q.n_tiles == 1 ? paged_blocks(q, 0) + kPagedTileCost : paged_units_before(q, q.n_tiles);
    PagedPlace p;
    p.seq = s;
    p.head = (u >> 31) == 0 && (per_head >> 31) == 0 ? (int)((uint32_t)u / (uint32_t)per_head) : (int)(u / per_head);
    u -= p.head * per_head;
    if (q.n_tiles == 1) {
        p.tile = 0;
        p.blk = min((int)u, paged_blocks(q, 0));
        return p;
    }
    int lo = 0, hi = q.n_tiles;  // units_before(lo) <= u < units_before(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (paged_units_before(q, mid) <= u) lo = mid; else hi = mid;
    }
    p.tile = lo;
    const int nb = paged_blocks(q, lo);
    p.blk = min((int)(u - paged_units_before(q, lo)), nb);  // (a boundary in the tile's cost is its end)
    if (q.kv > snap_keys) {
        const int step = (nb + 7) / 8;
        p.blk = min(nb, (p.blk + step / 2) / step * step);
    }
    return p;
}

struct PagedItem {
    int seq, head, q_row, n0, n1;  // tokens of the two contexts; n1 = 0: both contexts on the first's rows
    int lo, hi, nb;                // key tiles [lo, hi) of nb
    int pos, kv;                   // position of the first token; visible keys of the sequence
    __host__ __device__ bool dual() const { return n1 == 0; }
    // key tiles that context j takes: all, or every other one where both contexts have the same rows
    __host__ __device__ int steps(int j) const { return n1 == 0 ? (hi - lo + 1 - j) / 2 : hi - lo; }
    __host__ __device__ int tile(int j, int i) const { return n1 == 0 ? lo + 2 * i + j : lo + i; }
    __host__ __device__ bool partial() const { return lo > 0 || hi < nb; }
};

// Walks the items of a stretch; every role of a CTA walks the same ones.
struct PagedWalk {
    PagedPlace at, end;
    PagedSeq q;
    int loaded;
    __host__ __device__ PagedWalk(const PagedPlace& from, const PagedPlace& to) : at(from), end(to), loaded(-1) {}
    __host__ __device__ bool next(const PagedAttnArgs& a, PagedItem& it) {
        while (at.seq < a.c.batch) {
            if (loaded != at.seq) { q = paged_seq(a, at.seq); loaded = at.seq; }
            if (at.tile >= q.n_tiles) {
                at.tile = 0;
                if (++at.head >= a.c.H_kv || q.n_tiles == 0) {
                    if (at.seq >= end.seq) { at.seq = a.c.batch; return false; }
                    at.head = 0;
                    ++at.seq;
                }
                continue;
            }
            const int nb = paged_blocks(q, at.tile);
            const bool last = at.seq == end.seq && at.head == end.head && at.tile == end.tile;
            const int lo = at.blk, hi = last ? end.blk : nb, tile = at.tile, head = at.head, seq = at.seq;
            at.blk = 0;
            ++at.tile;
            if (last) at.seq = a.c.batch;
            if (lo >= hi) continue;
            const int first = tile * q.tile_tokens, n = min(q.tile_tokens, q.q_len - first);
            it.seq = seq; it.head = head;
            it.q_row = q.q_row + first;
            it.n0 = min(n, a.TPT); it.n1 = n - it.n0;
            it.lo = lo; it.hi = hi; it.nb = nb;
            it.pos = q.base + first; it.kv = q.kv;
            return true;
        }
        return false;
    }
};

// This CTA's stretch of the line into p.place: units of all sequences summed up, the boundaries looked up.  All threads
// call it; places are there after the caller's next __syncthreads.  (A third of a short call's time once: no 64-bit
// divisions where the numbers are small, warps without sequences stay out, the two places are worked out side by side.)
struct PagedPlan {
    int64_t scan[16], targets[2];
    PagedPlace place[2];
};

__device__ inline void paged_stretch(const PagedAttnArgs& a, PagedPlan& p, int64_t snap_keys, double inv_grid, int* status) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) p.targets[0] = p.targets[1] = -1;
    const int per = (a.c.batch + blockDim.x - 1) / blockDim.x;
    const int s_lo = min((int)threadIdx.x * per, a.c.batch), s_hi = min(s_lo + per, a.c.batch);
    const int busy = (a.c.batch + 32 * per - 1) / max(32 * per, 1);  // warps that have sequences
    int64_t mine = 0, upto = 0;
    if (warp < busy) {
        for (int s = s_lo; s < s_hi; ++s) {
            mine += paged_units(a, paged_seq(a, s));
            if (blockIdx.x == 0 && (a.c.kv_lens[s] < 0 || a.c.kv_lens[s] > paged_cap(a.c)))
                report_async(status, kAsyncBadIndex, 0x601);
        }
        upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t below = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += below;
        }
        if (lane == 31) p.scan[warp] = upto;
    }
    __syncthreads();
    if (warp < busy) {
        int64_t total = 0;
        for (int w = 0; w < busy; ++w) {
            if (w < warp) upto += p.scan[w];
            total += p.scan[w];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            // (the same rounding in every CTA, not decreasing; the last one is the end whatever it says)
            const int64_t target = (int64_t)((double)total * (double)(blockIdx.x + e) * inv_grid);
            if (blockIdx.x + e < gridDim.x && target >= upto - mine && target < upto) {  // (one thread)
                int64_t before = upto - mine;
                int s = s_lo;
                for (; s < s_hi - 1; ++s) {
                    const int64_t u = paged_units(a, paged_seq(a, s));
                    if (target < before + u) break;
                    before += u;
                }
                p.targets[e] = target - before;
                p.place[e].seq = s;
            }
        }
    }
    __syncthreads();
    if (lane == 0 && warp < 2)
        p.place[warp] = p.targets[warp] < 0 ? PagedPlace{a.c.batch, 0, 0, 0}
                                              : paged_place(a, p.place[warp].seq, p.targets[warp], snap_keys);
}

// ---------------------------------------------------------------- the kernel
struct PagedSmem {
    alignas(1024) uint8_t q[2][128 * 256];  // [context][d half][row][64 bf16]
    alignas(1024) uint8_t k[kPagedKStages][kPagedKeys * 256];  // [8 keys][d half][key][64 bf16]
    alignas(1024) uint8_t v[kPagedVStages][kPagedKeys * 256];
    float2 ml[128];                          // the second context's maxima and sums on their way to the first
    int8_t q_exp[2][2][128];                 // fp8: [item parity][context][row] power of two taken out of a row of Q
    alignas(8) uint64_t q_full[2], q_empty[2], q_land[2];
    uint64_t k_full[kPagedKStages], k_empty[kPagedKStages], k_land[kPagedKStages];
    uint64_t v_full[kPagedVStages], v_empty[kPagedVStages], v_land[kPagedVStages];
    uint64_t s_full[2], p_full[2][2], o_full[2], o_empty[2];  // [context], P: [half]
    uint64_t v_tail, ml_full, ml_empty, drain;
    PagedPlan plan;
    uint32_t tmem_base;
    int abort;
};

constexpr int paged_threads(bool f8) { return f8 ? 512 : 384; }

__device__ __forceinline__ uint32_t pack2_f16(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 bytes to a 16-byte boundary of global memory: one store where it is a 32-byte boundary too.
__device__ __forceinline__ void store32(void* to, const uint32_t* v) {
    if ((reinterpret_cast<uintptr_t>(to) & 31) == 0) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                     "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// Warps: 0-3 / 4-7 softmax of context 0 / 1 (thread = row), 8 loads K, 9 loads V, 10 issues the MMAs, 11 loads Q,
// 12-15 (fp8 caches) widen the tiles to fp16.
template <bool F8>
__global__ void __launch_bounds__(paged_threads(F8), 1)
paged_attn_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q1,
                     const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const PagedAttnArgs a, int box_keys, int64_t snap_keys, double inv_grid, int* status) {
    constexpr uint32_t TILE = F8 ? kPagedKeys * 128 : kPagedKeys * 256;  // bytes of a K or V tile in the cache
    extern __shared__ __align__(1024) uint8_t paged_smem[];  // (no room to round the base up)
    PagedSmem& sm = *reinterpret_cast<PagedSmem*>(paged_smem);
    if ((smem_u32(paged_smem) & 1023) != 0) {  // swizzled tiles need it; the same for every thread
        if (threadIdx.x == 0) {
            report_async(status, kAsyncBadIndex, 0x6FF);
            a.ends[blockIdx.x * 2] = make_int4(0, 0, 0, 0);  // (nothing to merge)
        }
        if constexpr (F8) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    if (F8 && a.min_len > 0) {  // paged_few8_kernel takes the shorter sequences, maybe all
        bool any = false;
        for (int s = threadIdx.x; s < a.c.batch; s += paged_threads(F8)) any |= a.c.cu_q[s + 1] - a.c.cu_q[s] >= a.min_len;
        if (__syncthreads_or(any) == 0) {
            if (threadIdx.x == 0) a.ends[blockIdx.x * 2] = make_int4(0, 0, 0, 0);
            asm volatile("griddepcontrol.wait;" ::: "memory");
            return;
        }
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort = &sm.abort;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.q_full[i], F8 ? 4 : 1); mbar_init(&sm.q_empty[i], 1); mbar_init(&sm.q_land[i], 1);
            mbar_init(&sm.s_full[i], 1); mbar_init(&sm.p_full[i][0], 4); mbar_init(&sm.p_full[i][1], 4);
            mbar_init(&sm.o_full[i], 1); mbar_init(&sm.o_empty[i], 4);
        }
        for (int i = 0; i < kPagedKStages; ++i) {
            mbar_init(&sm.k_full[i], F8 ? 4 : 1); mbar_init(&sm.k_empty[i], 1); mbar_init(&sm.k_land[i], 1);
        }
        for (int i = 0; i < kPagedVStages; ++i) {
            mbar_init(&sm.v_full[i], F8 ? 4 : 1); mbar_init(&sm.v_empty[i], 1); mbar_init(&sm.v_land[i], 1);
        }
        mbar_init(&sm.v_tail, 1); mbar_init(&sm.ml_full, 4); mbar_init(&sm.ml_empty, 4); mbar_init(&sm.drain, 1);
        sm.abort = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_q); tma_prefetch_desc(&tm_q1);
        tma_prefetch_desc(&tm_k); tma_prefetch_desc(&tm_v);
    }
    if (warp == 10) tmem_alloc(&sm.tmem_base, 512);

    paged_stretch(a, sm.plan, snap_keys, inv_grid, status);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    // Registers: the softmax warps hold a row of S (128) and more, the others little.  The shares stay within what the
    // block was launched with: 384 x 168 >= 256 x 192 + 128 x 120, 512 x 128 >= 256 x 176 + 2 x 128 x 80.
    // (Set at the head of each role: where roles share code the smallest share would rule.)
    constexpr int kRegsSoftmax = F8 ? 176 : 192, kRegsIssue = F8 ? 80 : 120, kRegsWiden = 80;
    PagedWalk walk(sm.plan.place[0], sm.plan.place[1]);
    PagedItem it{};

    if (warp >= 8 && warp < 12) {
        reg_release<kRegsIssue>();
        if (warp == 8 || warp == 9) {
            // ---------------- K / V producer: one box per page (or 128 keys of a larger one), a lane each
            const bool is_v = warp == 9;
            const int stages = is_v ? kPagedVStages : kPagedKStages;
            const int boxes = kPagedKeys / box_keys;
            const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
            const int nowhere = F8 ? a.c.n_pages * a.c.page_size : a.c.n_pages * a.c.page_size / 8;  // reads as zeros
            bool ok = true;
            int t = 0;
            uint32_t tails = 0;
            if (const long long late = g_debug_producer_delay; late > 0) spin_cycles(late);  // tests only
            // coordinate of this lane's box of key tile b: its page's row, or outside the pool
            auto place_of = [&](int b) {
                const uint32_t key = (uint32_t)b * kPagedKeys + lane * box_keys, size = a.c.page_size;  // (below 2^31 + 128)
                if (lane >= boxes || key >= (uint32_t)it.kv) return nowhere;
                const uint32_t slot = key / size;
                const int page = a.c.table[(int64_t)it.seq * a.c.max_pages + slot];
                if (page < 0 || page >= a.c.n_pages) {
                    report_async(status, kAsyncBadIndex, 0x602);
                    return nowhere;
                }
                const int row = page * a.c.page_size + (int)(key - slot * size);
                return F8 ? row : row / 8;
            };
            while (ok && walk.next(a, it)) {
                int where = place_of(it.lo);
                for (int b = it.lo; b < it.hi; ++b, ++t) {
                    const int where_next = b + 1 < it.hi ? place_of(b + 1) : 0;
                    const int st = t % stages;
                    const uint32_t use = t / stages;
                    uint64_t* empty = is_v ? &sm.v_empty[st] : &sm.k_empty[st];
                    uint64_t* full = is_v ? &sm.v_full[st] : &sm.k_full[st];
                    uint64_t* land = is_v ? &sm.v_land[st] : &sm.k_land[st];
                    uint8_t* dst = is_v ? sm.v[st] : sm.k[st];
                    if (use > 0 && !mbar_wait(empty, (use - 1) & 1, abort)) {
                        if (lane == 0) report_async(status, kAsyncTimeout, 0x611);
                        ok = false;
                        break;
                    }
                    // The last tile's V rows behind the end may hold anything, and 0 * NaN is NaN: they are overwritten
                    // with zeros before the MMA sees the tile (fp8: by the widening warps).
                    const int rows = it.kv - b * kPagedKeys;  // rows inside the sequence
                    const bool tail = !F8 && is_v && rows < kPagedKeys;
                    uint64_t* bar = F8 ? land : (tail ? &sm.v_tail : full);
                    if (lane == 0) mbar_arrive_expect_tx(bar, TILE);
                    __syncwarp();
                    if (lane < boxes) {
                        // (fp8: 32 keys into the upper half of the 8 KB of their fp16)
                        if constexpr (F8) tma_load_3d(dst + (lane * box_keys >> 5) * 8192 + 4096 + (lane * box_keys & 31) * 128, tm, 0, it.head, where, bar);
                        else tma_load_5d(dst + lane * box_keys * 256, tm, 0, 0, 0, it.head, where, bar);
                    }
                    if (tail) {
                        if (!mbar_wait(&sm.v_tail, tails & 1, abort)) {
                            if (lane == 0) report_async(status, kAsyncTimeout, 0x612);
                            ok = false;
                            break;
                        }
                        ++tails;
                        for (int i = max(rows, 0) * 16 + lane; i < kPagedKeys * 16; i += 32) {
                            const int key = i >> 4, c = i & 15;
                            *reinterpret_cast<uint4*>(dst + (key >> 3) * 2048 + (c >> 3) * 1024 + (key & 7) * 128 + (c & 7) * 16) =
                                make_uint4(0u, 0u, 0u, 0u);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full);
                    }
                    where = where_next;
                }
            }
            if (*abort != 0) spin_cycles(200000);
        } else if (warp == 11) {
            // ---------------- Q producer, and the note for the merge
            PagedEnds e{};
            bool ok = true;
            uint32_t used[2] = {0, 0};
            while (walk.next(a, it)) {
                if (e.first == 0) e.first = it.lo == 0 ? 3 : (it.hi < it.nb ? 1 : 2);
                e.open = it.lo == 0 && it.hi < it.nb;
                e.q_row = it.q_row; e.tokens = it.n0 + it.n1; e.head = it.head;
                for (int j = 0; j < 2 && ok; ++j) {
                    const int n = j == 0 ? it.n0 : it.n1;
                    if (n == 0) continue;
                    if (used[j] > 0 && !mbar_wait(&sm.q_empty[j], (used[j] - 1) & 1, abort)) {
                        if (lane == 0) report_async(status, kAsyncTimeout, 0x621);
                        ok = false;
                        break;
                    }
                    ++used[j];
                    const int row = it.q_row + j * a.TPT, head = it.head * a.G;
                    // Few tokens: their own boxes (rows behind them keep what they held: no row reads another's).  All: one
                    // box for each half of d; tokens of the next sequence come along, tokens that are not there read as zeros.
                    const bool few = n * 2 <= 16 && n < a.TPT && a.G % 8 == 0;
                    uint64_t* bar = F8 ? &sm.q_land[j] : &sm.q_full[j];
                    if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)((few ? n : a.TPT) * a.G * 256));
                    __syncwarp();
                    if (few) {
                        if (lane < 2 * n)
                            tma_load_3d(sm.q[j] + (lane & 1) * 16384 + (lane >> 1) * a.G * 128, &tm_q1, (lane & 1) * 64, head, row + (lane >> 1),
                                        bar);
                    } else if (lane < 2) {
                        tma_load_3d(sm.q[j] + lane * 16384, &tm_q, lane * 64, head, row, bar);
                    }
                }
            }
            if (lane == 0) {
                a.ends[blockIdx.x * 2] = make_int4(e.first, e.open, e.q_row, e.tokens);
                a.ends[blockIdx.x * 2 + 1] = make_int4(e.head, 0, 0, 0);
            }
            if (*abort != 0) spin_cycles(200000);
        } else if (warp == 10) {
            // ---------------- MMA issuer: S_j(i) = Q_j K^T, then, once P_j(i) is written over it, O_j += P_j(i) V.
            // S_j(i+1) is issued right behind O_j += P_j(i) V: MMAs run in issue order, so it may overwrite P_j(i), it runs
            // while the other context's softmax is at work, and the barrier that says S_j(i) is there says as well that O_j
            // holds all steps before.  P comes in halves, so that the product starts on the first.  (S in two 64-key
            // buffers, one product ahead, was slower: 64-key products read Q twice as often, and shared memory is what the
            // MMAs run short of; 128-row chunk 4.8 against 4.3 ms.)
            // The whole warp walks and waits, one elected lane issues: descriptors then stay in uniform registers.
            constexpr uint32_t idesc = F8 ? make_idesc_f16(128, 128, false, false) : make_idesc_bf16(128, 128, false, false);
            constexpr uint32_t idesc_o = F8 ? make_idesc_f16(128, 128, false, true) : make_idesc_bf16(128, 128, false, true);
            constexpr uint32_t kTile = kPagedKeys * 256 / 16;  // in descriptor units of 16 bytes
            const uint64_t q_desc = make_smem_desc(smem_u32(sm.q[0]), 16, 1024), k_desc = make_smem_desc(smem_u32(sm.k[0]), 16, 2048);
            // V as the MN-major B operand: 8-key groups 2 KB apart, the other 64 columns of d 1 KB away
            const uint64_t v_desc = make_smem_desc(smem_u32(sm.v[0]), 1024, 2048);
            uint32_t n_p[2] = {0, 0}, n_o[2] = {0, 0}, n_q[2] = {0, 0};  // P's, items and uses of Q so far
            uint32_t ks = 0, k_phase = 0, vs = 0, v_phase = 0;            // stage of the next K / V tile and its use's parity
            bool ok = true;
            while (ok && walk.next(a, it)) {
                const bool dual = it.dual();
                const int st[2] = {it.steps(0), it.steps(1)};
                for (int i = -1; ok && i < st[0]; ++i) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t ts = tmem + j * 128, to = tmem + 256 + j * 128;
                        const bool first_user = dual || j == 0, last_user = dual || j == 1;  // of a K or V tile
                        // (K is waited for behind the product with V: where loads are the limit, V's stage is free sooner)
                        if (i >= 0 && i < st[j]) {
                            if ((first_user && !mbar_wait(&sm.v_full[vs], v_phase, abort)) ||
                                (i == 0 && n_o[j] > 0 && !mbar_wait(&sm.o_empty[j], (n_o[j] - 1) & 1, abort)) ||
                                !mbar_wait(&sm.p_full[j][0], n_p[j] & 1, abort)) {
                                if (lane == 0) report_async(status, kAsyncTimeout, 0x631);
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            const uint64_t vd = v_desc + vs * kTile;
                            if (elect_one()) {
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk) mma_bf16_ts(to, ts + kk * 8, vd + (uint64_t)(kk * 256), idesc_o, i > 0 || kk > 0);
                            }
                            __syncwarp();
                            if (!mbar_wait(&sm.p_full[j][1], n_p[j]++ & 1, abort)) {
                                if (lane == 0) report_async(status, kAsyncTimeout, 0x632);
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int kk = 4; kk < 8; ++kk) mma_bf16_ts(to, ts + kk * 8, vd + (uint64_t)(kk * 256), idesc_o, true);
                                if (last_user) mma_commit(&sm.v_empty[vs]);
                                if (i == st[j] - 1) mma_commit(&sm.o_full[j]);
                            }
                            __syncwarp();
                            n_o[j] += i == st[j] - 1;
                            if (last_user && ++vs == kPagedVStages) { vs = 0; v_phase ^= 1; }
                        }
                        if (i + 1 < st[j]) {
                            const int qb = dual ? 0 : j;
                            if ((first_user && !mbar_wait(&sm.k_full[ks], k_phase, abort)) ||
                                (i == -1 && (!dual || j == 0) && !mbar_wait(&sm.q_full[qb], n_q[qb] & 1, abort))) {
                                if (lane == 0) report_async(status, kAsyncTimeout, 0x633);
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            const bool q_done = dual ? 2 * (i + 1) + j == it.hi - it.lo - 1 : i + 2 == st[j];
                            if (elect_one()) {
                                const uint64_t qd = q_desc + qb * (128 * 256 / 16), kd = k_desc + ks * kTile;
#pragma unroll
                                for (int kk = 0; kk < 8; ++kk)  // 16 of d each; second half of Q 16 KB on, of K 1 KB
                                    mma_bf16_ss(ts, qd + (uint64_t)((kk >> 2) * 1024 + 2 * (kk & 3)),
                                                kd + (uint64_t)((kk >> 2) * 64 + 2 * (kk & 3)), idesc, kk > 0);
                                mma_commit(&sm.s_full[j]);
                                if (last_user) mma_commit(&sm.k_empty[ks]);
                                if (q_done) mma_commit(&sm.q_empty[qb]);
                            }
                            __syncwarp();
                            if (last_user && ++ks == kPagedKStages) { ks = 0; k_phase ^= 1; }
                        }
                    }
                }
                ++n_q[0];
                n_q[1] += !dual;
            }
            if (*abort != 0) {
                if (elect_one()) mma_commit(&sm.drain);
                __syncwarp();
                mbar_wait_quiet(&sm.drain, 0, 20000000);
            }
        }
    } else if (warp >= 12) {
        // ---------------- widening (fp8): K and V become fp16, which holds every E4M3 value and takes one conversion
        // for two elements (bf16 takes four operations).  Warp w widens keys 32w .. 32w+31 of every tile: their 4 KB (row =
        // key, 128 bytes, chunks swizzled by key mod 8) land in the upper half of the 8 KB that their fp16 will fill, so
        // that a warp overwrites only what it has read itself.  The fence that shows a tile to the MMAs waits for the
        // warp's stores, hundreds of cycles; it comes behind the next tile's loads unless that tile is late.
        // Q becomes fp16 as well, with a power of two taken out of each row so that any bf16 row fits: what is rounded
        // off is below 2^-38 of the row's largest element.  The softmax warps put it back into the scale.
        if constexpr (F8) {
            reg_release<kRegsWiden>();
            const int w = warp - 12, key = w * 32 + lane, sw = lane & 7;
            const uint32_t from = w * 8192 + 4096 + lane * 128, into = w * 8192 + (lane >> 3) * 2048 + sw * 128;
            uint32_t t = 0, n_q[2] = {0, 0}, item = 0;
            uint64_t* written = nullptr;  // the barrier of the tile that is written and not yet shown
            auto show = [&]() {
                if (written == nullptr) return;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(written);
                written = nullptr;
            };
            bool ok = true;
            while (ok && walk.next(a, it)) {
                for (int b = it.lo; ok && b < it.hi; ++b, ++t) {
                    for (int kv = 0; kv < 2; ++kv) {
                        const uint32_t stages = kv == 0 ? kPagedKStages : kPagedVStages, st = t % stages;
                        uint8_t* tile = kv == 0 ? sm.k[st] : sm.v[st];
                        uint64_t* land = kv == 0 ? &sm.k_land[st] : &sm.v_land[st];
                        if (!__all_sync(0xffffffffu, mbar_try_wait(land, (t / stages) & 1))) {
                            show();  // (what has to be seen for this tile to come)
                            if (!mbar_wait(land, (t / stages) & 1, abort)) {
                                if (lane == 0) report_async(status, kAsyncTimeout, 0x641);
                                ok = false;
                                break;
                            }
                        }
                        // (rows behind the end may hold anything, and 0 * NaN is NaN: V's become zeros)
                        const bool inside = kv == 0 || (int64_t)b * kPagedKeys + key < it.kv;
                        uint4 x[8];
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            x[c] = make_uint4(0u, 0u, 0u, 0u);
                            if (inside) x[c] = *reinterpret_cast<const uint4*>(tile + from + ((c ^ sw) << 4));
                        }
                        show();
                        __syncwarp();  // (every lane has read its row)
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            uint4 lo, hi;
                            e4m3x4_to_f16x2x2(x[c].x, lo.x, lo.y); e4m3x4_to_f16x2x2(x[c].y, lo.z, lo.w);
                            e4m3x4_to_f16x2x2(x[c].z, hi.x, hi.y); e4m3x4_to_f16x2x2(x[c].w, hi.z, hi.w);
                            const int cc = 2 * (c & 3);
                            uint8_t* to = tile + into + (c >> 2) * 1024;
                            *reinterpret_cast<uint4*>(to + ((cc ^ sw) << 4)) = lo;
                            *reinterpret_cast<uint4*>(to + (((cc + 1) ^ sw) << 4)) = hi;
                        }
                        written = kv == 0 ? &sm.k_full[st] : &sm.v_full[st];
                    }
                    for (int j = 0; ok && b == it.lo && j < (it.dual() ? 1 : 2); ++j) {  // Q, behind the first tile
                        show();
                        if (!mbar_wait(&sm.q_land[j], n_q[j]++ & 1, abort)) {
                            if (lane == 0) report_async(status, kAsyncTimeout, 0x642);
                            ok = false;
                            break;
                        }
                        uint8_t* row = sm.q[j] + key * 128;  // thread = row: two halves of 128 bytes
                        uint32_t most = 0;
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            const uint4 v = *reinterpret_cast<const uint4*>(row + (c >> 3) * 16384 + (((c & 7) ^ sw) << 4));
                            most = max(max(max(most, v.x & 0x7FFF0000u), max(v.y & 0x7FFF0000u, v.z & 0x7FFF0000u)), v.w & 0x7FFF0000u);
                            most = max(max(max(most, v.x << 17 >> 1), max(v.y << 17 >> 1, v.z << 17 >> 1)), v.w << 17 >> 1);
                        }
                        // the largest element goes to [2^14, 2^15): beyond, for rows below 2^-98, as far as 2^112 takes it
                        const int e = most == 0 ? 0 : max((int)(most >> 23) - 127 - 14, -112);
                        const float f = __uint_as_float((uint32_t)(127 - e) << 23);
                        sm.q_exp[item & 1][j][key] = (int8_t)e;
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            uint4* at = reinterpret_cast<uint4*>(row + (c >> 3) * 16384 + (((c & 7) ^ sw) << 4));
                            const F8v y = widen8(*at);
                            *at = make_uint4(pack2_f16(y.v[0].x * f, y.v[0].y * f), pack2_f16(y.v[1].x * f, y.v[1].y * f),
                                             pack2_f16(y.v[2].x * f, y.v[2].y * f), pack2_f16(y.v[3].x * f, y.v[3].y * f));
                        }
                        written = &sm.q_full[j];
                        show();
                    }
                }
                ++item;
            }
            show();
        }
    } else {
        reg_acquire<kRegsSoftmax>();
        // ---------------- softmax and epilogue: thread = row (TMEM lane)
        const int j = warp >> 2, quarter = warp & 3;
        const int row = quarter * 32 + lane, tok = row / a.G, g = row - tok * a.G;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tmem_s = tmem + lane_base + j * 128, tmem_o = tmem + lane_base + 256 + j * 128;
        const int H_q = a.c.H_kv * a.G;
        uint32_t n_s = 0, n_o[2] = {0, 0}, n_ml = 0;  // steps, accumulators of the two contexts, merges so far
        bool ok = true;
        uint32_t n_item = 0;
        for (; ok && walk.next(a, it); ++n_item) {
            const bool dual = it.dual();
            const int steps = it.steps(j);
            const int tokens = dual || j == 0 ? it.n0 : it.n1;
            const bool warp_on = quarter * 32 < tokens * a.G;  // some row of the warp is a query's
            const bool row_on = tok < tokens;
            const int first = dual || j == 0 ? 0 : a.TPT;
            const int64_t pos = (int64_t)it.pos + first + tok;
            float m_ref = -INFINITY, l = 0.f, scale = a.scale_log2e;
            for (int i = 0; i < steps; ++i) {
                if (!mbar_wait(&sm.s_full[j], n_s++ & 1, abort)) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x651);
                    ok = false;
                    break;
                }
                if (!warp_on) {
                    if (lane < 2) mbar_arrive(&sm.p_full[j][lane]);
                    continue;
                }
                tc_fence_after();
                if (F8 && i == 0) scale *= __uint_as_float((uint32_t)(127 + sm.q_exp[n_item & 1][dual ? 0 : j][row]) << 23);
                uint32_t sv[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_32x32(tmem_s + c * 32, sv[c]);
                tmem_wait_ld();
                // keys 0..lim of the tile are visible
                const int lim = (int)max(min(pos - (int64_t)it.tile(j, i) * kPagedKeys, (int64_t)kPagedKeys), (int64_t)-1);
                if (lim < kPagedKeys - 1) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e > lim) sv[c][e] = 0xFF800000u;  // -inf
                }
                const float mx = fmaxf(fmaxf(tree_max32(sv[0]), tree_max32(sv[1])), fmaxf(tree_max32(sv[2]), tree_max32(sv[3])));
                // The reference maximum moves only when a row's maximum has outgrown it by 2^kPGrow, so that O is hardly
                // ever rescaled.  bf16 P keeps its relative precision at any size.  fp16 P is held 2^10 up, which leaves
                // 2^5 to grow below its largest value and rounds by 2^-11 of the value or 2^-35 of the row's largest.
                constexpr float kPGrow = F8 ? 5.f : 8.f, kPShift = F8 ? 10.f : 0.f;
                const float m_new = fmaxf(m_ref, mx);
                if (i == 0) {
                    m_ref = m_new;
                } else if (__any_sync(0xffffffffu, row_on && (m_new - m_ref) * scale > kPGrow)) {
                    const float corr = m_new == -INFINITY ? 1.f : ex2_approx((m_ref - m_new) * scale);
                    m_ref = m_new;
                    l *= corr;
#pragma unroll 1
                    for (int c = 0; c < 8; ++c) {
                        uint32_t ov[16];
                        tmem_ld_32x16(tmem_o + c * 16, ov);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * corr);
                        tmem_st_32x16(tmem_o + c * 16, ov);
                    }
                }
                const float mc = m_ref == -INFINITY ? 0.f : fmaf(m_ref, scale, -kPShift);
                const float2 sc2 = make_float2(scale, scale), mc2 = make_float2(-mc, -mc);
                float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t pk[32];
#pragma unroll
                    for (int w = 0; w < 32; ++w) {
                        const uint32_t* from = &sv[2 * h + (w >> 4)][2 * (w & 15)];
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(from[0]), __uint_as_float(from[1])), sc2, mc2);
                        const float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        l2[w & 1] = __fadd2_rn(l2[w & 1], p);
                        pk[w] = F8 ? pack2_f16(p.x, p.y) : pack2(p.x, p.y);
                    }
                    tmem_st_32x32(tmem_s + h * 32, pk);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.p_full[j][h]);
                }
                l += (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
            }
            if (!ok) break;
            const float m_log2 = m_ref == -INFINITY ? -INFINITY : fmaf(m_ref, scale, F8 ? -10.f : -0.f);
            const bool merge = dual && it.steps(1) > 0;
            if (dual && j == 1) {
                // hand the row's maximum and sum to the first context, which reads O_1 as well
                if (!merge) continue;
                if (n_ml > 0 && !mbar_wait(&sm.ml_empty, (n_ml - 1) & 1, abort)) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x652);
                    break;
                }
                ++n_ml; ++n_o[1];
                sm.ml[row] = make_float2(m_log2, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.ml_full);
                continue;
            }
            float w0 = 1.f, w1 = 0.f, m_all = m_log2;
            if (!mbar_wait(&sm.o_full[j], n_o[j] & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x653);
                break;
            }
            if (merge) {
                // (O_1 of the item before was complete before this item's first S was issued: the parity is this item's)
                if (!mbar_wait(&sm.o_full[1], n_o[1] & 1, abort) || !mbar_wait(&sm.ml_full, n_ml & 1, abort)) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x654);
                    break;
                }
                ++n_ml;
                const float2 ml = sm.ml[row];
                m_all = fmaxf(m_log2, ml.x);
                w0 = m_log2 == -INFINITY ? 0.f : ex2_approx(m_log2 - m_all);
                w1 = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - m_all);
                l = w0 * l + w1 * ml.y;
            }
            n_o[0] += 1;
            n_o[1] += !dual || merge;
            tc_fence_after();
            if (warp_on) {
                const bool partial = it.partial();
                const int64_t out_row = ((int64_t)it.q_row + first + tok) * H_q + it.head * a.G + g;
                const int64_t slot_row = ((int64_t)blockIdx.x * 2 + (it.lo > 0 ? 0 : 1)) * a.slot_rows + (first > 0 ? 128 : 0) + row;
                if (!partial) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing is zero)
                    w0 *= inv; w1 *= inv;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t ov[32];
                    tmem_ld_32x32(tmem_o + c * 32, ov);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * w0);
                    if (merge) {
                        uint32_t o1[32];
                        tmem_ld_32x32(tmem_o + 128 + c * 32, o1);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(fmaf(__uint_as_float(o1[e]), w1, __uint_as_float(ov[e])));
                    }
                    // (32 bytes a store: whole sectors, where the lanes' rows are 256 bytes and more apart)
                    if (row_on && partial) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(a.part_o + slot_row * 128 + c * 32 + e * 8, &ov[8 * e]);
                    } else if (row_on) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = pack2(__uint_as_float(ov[2 * e]), __uint_as_float(ov[2 * e + 1]));
                        store32(a.out + out_row * 128 + c * 32, pk);
                        store32(a.out + out_row * 128 + c * 32 + 16, pk + 8);
                    }
                    __syncwarp();
                }
                if (row_on) {
                    if (partial) a.part_ml[slot_row] = make_float2(m_all, l);
                    else if (a.lse != nullptr) a.lse[out_row] = l == 0.f ? -INFINITY : (m_all + log2f(l)) * 0.6931471805599453f;
                }
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&sm.o_empty[j]);
                if (merge) { mbar_arrive(&sm.o_empty[1]); mbar_arrive(&sm.ml_empty); }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 10) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    // Launched early behind paged_few8_kernel, if that takes part: the merge waits for this kernel only, which therefore ends
    // after that one.
    if constexpr (F8) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Merges the partials of tiles that stretch boundaries cut: CTA (i, .) the tile that attention CTA i left open, a warp
// per row.  With M the largest reference maximum, O = sum 2^(m - M) O_p, l likewise; out = O / l.  The order of the
// parts is that of the line, so equal calls give equal bits.  BOTH: one launch merges for both attention kernels of a call on
// an fp8 cache, the first CTAs the tiles cut in c0, the others those of c1 (choosing between them costs 0.5 us, so other calls
// do without).
constexpr int kMergeThreads = 128, kMergeWarps = kMergeThreads / 32;
struct PagedCuts {  // of one attention kernel; the members as in PagedAttnArgs
    const float* part_o;
    const float2* part_ml;
    const int4* ends;
    int TPT, slot_rows, n_ctas;
};

template <bool BOTH>
__global__ void __launch_bounds__(kMergeThreads)
paged_combine_kernel(const PagedAttnArgs a, const PagedCuts c0, const PagedCuts c1) {
    const bool other = BOTH && (int)blockIdx.x >= c0.n_ctas;
    const int cta = other ? blockIdx.x - c0.n_ctas : blockIdx.x, n_ctas = other ? c1.n_ctas : c0.n_ctas;
    const int4* ends = other ? c1.ends : c0.ends;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched early: what the attention kernels wrote is there after this
    const int4 e = ends[cta * 2];
    if (e.y == 0) return;
    const int TPT = other ? c1.TPT : c0.TPT, slot_rows = other ? c1.slot_rows : c0.slot_rows;
    const float* part_o = other ? c1.part_o : c0.part_o;
    const float2* part_ml = other ? c1.part_ml : c0.part_ml;
    const int head = ends[cta * 2 + 1].x, tokens = e.w, lane = threadIdx.x & 31;
    __shared__ int s_slot[512];  // parts: at most one for each CTA
    __shared__ int s_n;
    if (threadIdx.x < 32) {
        int n = 1;
        if (lane == 0) s_slot[0] = 2 * cta + 1;
        for (int c = cta + 1; c < n_ctas; c += 32) {
            const int first = c + lane < n_ctas ? ends[(c + lane) * 2].x : 3;
            const unsigned stop = __ballot_sync(0xffffffffu, first >= 2);  // 2: the last part, 3: none of this tile's
            const int upto = stop ? __ffs(stop) - 1 : 32;
            const bool part = (lane < upto && first == 1) || (lane == upto && first == 2);
            const unsigned parts = __ballot_sync(0xffffffffu, part);
            if (part) s_slot[n + __popc(parts & ((1u << lane) - 1))] = 2 * (c + lane);
            n += __popc(parts);
            if (stop) break;
        }
        if (lane == 0) s_n = n;
    }
    __syncthreads();
    const int n = s_n, rows = tokens * a.G, H_q = a.c.H_kv * a.G;
    for (int r = blockIdx.y * kMergeWarps + (threadIdx.x >> 5); r < rows; r += gridDim.y * kMergeWarps) {
        const int tok = r / a.G, g = r - tok * a.G;
        const int in_slot = tok < TPT ? r : 128 + (tok - TPT) * a.G + g;
        float M = -INFINITY;
        for (int p = lane; p < n; p += 32) M = fmaxf(M, part_ml[(int64_t)s_slot[p] * slot_rows + in_slot].x);
        M = warp_max(M);
        float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = 0; p < n; ++p) {
            const int64_t at = (int64_t)s_slot[p] * slot_rows + in_slot;
            const float2 ml = part_ml[at];
            const float4 x = *reinterpret_cast<const float4*>(part_o + at * 128 + lane * 4);
            const float w = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - M);
            L = fmaf(w, ml.y, L);
            o[0] = fmaf(w, x.x, o[0]); o[1] = fmaf(w, x.y, o[1]); o[2] = fmaf(w, x.z, o[2]); o[3] = fmaf(w, x.w, o[3]);
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int64_t row = ((int64_t)e.z + tok) * H_q + head * a.G + g;
        *reinterpret_cast<uint2*>(a.out + row * 128 + lane * 4) = make_uint2(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv));
        if (lane == 0 && a.lse != nullptr) a.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    }
}

// ---------------------------------------------------------------- other shapes
// Head sizes, page sizes and group sizes the kernel above does not take: a warp per (token, query head), 32 keys at a
// time (a lane each for the products, then all lanes on d for the values).  fp32 throughout.
template <bool F8>
__global__ void __launch_bounds__(128)
paged_attn_generic_kernel(PagedAttnArgs a, const __nv_bfloat16* __restrict__ q, const void* __restrict__ k_pool,
                          const void* __restrict__ v_pool, int d, int* status) {
    __shared__ float qs[4][256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int H_q = a.c.H_kv * a.G;
    const int64_t unit = (int64_t)blockIdx.x * 4 + warp;
    if (unit >= (int64_t)a.n_tokens * H_q) return;
    const int i = (int)(unit / H_q), h = (int)(unit - (int64_t)i * H_q), hk = h / a.G;
    const int s = paged_seq_of(a.c, i);
    if (s < 0) return;
    const int64_t cap = paged_cap(a.c);
    const int len = a.c.kv_lens[s];
    if ((len < 0 || len > cap) && lane == 0) report_async(status, kAsyncBadIndex, 0x601);
    const int64_t kv = min((int64_t)max(len, 0), cap);
    const int64_t pos = kv - (a.c.cu_q[s + 1] - i);
    for (int c = lane; c < d; c += 32) qs[warp][c] = __bfloat162float(q[unit * d + c]) * a.scale_log2e;
    __syncwarp();
    float m = -INFINITY, l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t j0 = 0; j0 <= pos; j0 += 32) {
        const int64_t key = j0 + lane;
        int64_t row = -1;
        if (key <= pos) {
            const int page = a.c.table[(int64_t)s * a.c.max_pages + key / a.c.page_size];
            if (page >= 0 && page < a.c.n_pages) row = ((int64_t)page * a.c.page_size + key % a.c.page_size) * a.c.H_kv + hk;
            else report_async(status, kAsyncBadIndex, 0x602);
        }
        float x = -INFINITY;
        if (row >= 0) {
            x = 0.f;
            for (int c = 0; c < d; ++c) x = fmaf(qs[warp][c], idx_elem<F8>(static_cast<const uint8_t*>(k_pool) + row * d * (F8 ? 1 : 2), c), x);
        }
        const float m_new = fmaxf(m, warp_max(x));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float corr = m == -INFINITY ? 0.f : exp2f(m - m_use);
        const float p = row >= 0 ? exp2f(x - m_use) : 0.f;
        l = l * corr + warp_sum(p);
        m = m_new;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[c] *= corr;
        for (int t = 0; t < 32; ++t) {
            const int64_t rt = __shfl_sync(0xffffffffu, row, t);
            const float pt = __shfl_sync(0xffffffffu, p, t);
            if (rt < 0) continue;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (lane + 32 * c < d) o[c] = fmaf(pt, idx_elem<F8>(static_cast<const uint8_t*>(v_pool) + rt * d * (F8 ? 1 : 2), lane + 32 * c), o[c]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (lane + 32 * c < d) a.out[unit * d + lane + 32 * c] = __float2bfloat16(o[c] * inv);
    if (lane == 0 && a.lse != nullptr) a.lse[unit] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace msa
