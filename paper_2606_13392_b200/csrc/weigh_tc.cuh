// The attention weight that cached tokens receive (see weigh.cuh), for sequences of more than a few query rows: tcgen05.
//
// Keys are the rows of the products, D = K Q^T, so that the sum over queries runs along a row of the accumulator: a thread
// owns a key, adds exp2(scale D - lse) over the columns, and nothing is exchanged until a part ends.  256 keys (two
// operand tiles) stay in shared memory while the queries' tiles of 128 rows - (token, head of the group) pairs, TPT = 128 / G
// tokens - stream past them; each tile is read once for two products.
// One exponential for 2 * 128 flops: bound by the exponential unit (16 a cycle and SM; 4096 tokens on 28K have 8 10^9, 1.8 ms of
// it at 1.9 GHz) at the clock that the board's power allows.
// Measured (64/8 heads): 4096 tokens on 28K 2.36 - 2.46 ms, 0.84 - 0.87 PFLOP/s; on themselves 170 us; 512 on 7K 80 - 90 us; the
// last 32 of 4 prompts of 8K - 16K 45 us; the last 17 - 48 of 6 prompts of up to 32K on fp8, 64/4 heads, 139 us.
// Looked at and not kept: the keys as operands in tensor memory (2.40 ms; windows 139 -> 165 us, the next keys wait for the last
// products), without exponentials 1.95 ms, without anything but the products 1.65 ms (power), with loops that share code 2.58 ms.
//
// Unit of work: one tile of rows against 256 keys of a (sequence, KV head).  All units form one line (sequence, head, key
// block, tile), tiles that see none of the keys left out; every CTA takes an equal stretch, so that neither ragged batches nor the
// causal triangle leave CTAs idle.  A key block that a boundary cuts leaves partial sums (at most two per CTA), which
// weigh_merge_kernel adds up in order (no atomics: equal calls give equal bits).
#pragma once

#include "paged_attn.cuh"
#include "weigh.cuh"

namespace msa {

constexpr int kWtKeys = 256, kWtStages = 3;
constexpr int kWtEpiWarps = 16, kWtWidenWarps = 4;
constexpr int weigh_tc_threads(bool f8) { return (kWtEpiWarps + 4 + (f8 ? kWtWidenWarps : 0)) * 32; }
constexpr int kWtBlockCost = 2;  // tiles' worth of a key block's beginning and end

// kb0: first key block behind `base`; [kb_lim, n_kb): blocks that no row of the call sees (it may lack rows)
struct WeighTcSeq { int q_row, q_len, kv, base, n_tiles, kb0, kb_lim, n_kb; };

__host__ __device__ __forceinline__ WeighTcSeq weigh_tc_seq(const WeighArgs& a, int TPT, int s) {
    WeighTcSeq q;
    const int lo = max(a.c.cu_q[s], 0), end = a.c.cu_q[s + 1], hi = min(end, a.n_tokens);
    q.q_row = lo;
    q.q_len = max(hi - lo, 0);
    if (q.q_len < a.min_len || q.q_len > a.max_len) q.q_len = 0;
    q.kv = (int)min((int64_t)max(a.c.kv_lens[s], 0), paged_places(a.c));
    q.base = q.kv - max(end - lo, 0);
    q.n_tiles = (q.q_len + TPT - 1) / TPT;
    q.n_kb = q.q_len == 0 ? 0 : (int)(((int64_t)q.kv + kWtKeys - 1) / kWtKeys);
    q.kb0 = q.base <= 0 ? 0 : (int)min(((int64_t)q.base + kWtKeys - 1) / kWtKeys, (int64_t)q.n_kb);
    q.kb_lim = (int)min((max((int64_t)q.base + (int64_t)q.n_tiles * TPT, (int64_t)0) + kWtKeys - 1) / kWtKeys, (int64_t)q.n_kb);
    return q;
}

// First tile with a token that sees a key of block kb (n_tiles where the call lacks those rows).
__host__ __device__ __forceinline__ int weigh_tc_first(const WeighTcSeq& q, int TPT, int kb) {
    const int64_t tok = (int64_t)kb * kWtKeys - q.base;
    return tok <= 0 ? 0 : (int)min((uint32_t)tok / (uint32_t)TPT, (uint32_t)q.n_tiles);  // (lengths are below 2^31)
}

// Units of the first kb key blocks of one head, their cost included.
__host__ __device__ inline int64_t weigh_tc_before(const WeighTcSeq& q, int TPT, int kb) {
    const int seen = min(kb, q.kb_lim), extra = max(seen - q.kb0, 0);
    int64_t u = (int64_t)seen * q.n_tiles + (int64_t)kb * kWtBlockCost;
    if (extra > 0) u -= floor_sum(extra, TPT, kWtKeys, (int64_t)q.kb0 * kWtKeys - q.base);
    return u;
}

struct WeighTcSpot { int seq, head, kb, tile; };

struct WeighPart {
    int seq, head, kb, q_row, q_len, kv, base;
    int t0, lo, hi, n;  // tiles [lo, hi) of the block's [t0, n)
    __device__ bool whole() const { return lo == t0 && hi == n; }
};

struct WeighTcWalk {
    WeighTcSpot at, end;
    WeighTcSeq q;
    int loaded;
    __device__ WeighTcWalk(const WeighTcSpot& from, const WeighTcSpot& to) : at(from), end(to), loaded(-1) {}
    __device__ bool next(const WeighArgs& a, int TPT, WeighPart& p) {
        while (at.seq < a.c.batch) {
            if (loaded != at.seq) { q = weigh_tc_seq(a, TPT, at.seq); loaded = at.seq; }
            if (at.kb >= q.n_kb) {
                at.kb = 0;
                if (++at.head >= a.c.H_kv || q.n_kb == 0) {
                    if (at.seq >= end.seq) { at.seq = a.c.batch; return false; }
                    at.head = 0;
                    ++at.seq;
                }
                at.tile = 0;
                continue;
            }
            const bool last = at.seq == end.seq && at.head == end.head && at.kb == end.kb;
            const int t0 = weigh_tc_first(q, TPT, at.kb), lo = max(at.tile, t0), hi = last ? min(end.tile, q.n_tiles) : q.n_tiles;
            p = WeighPart{at.seq, at.head, at.kb, q.q_row, q.q_len, q.kv, q.base, t0, lo, hi, q.n_tiles};
            at.tile = 0;
            ++at.kb;
            if (last) at.seq = a.c.batch;
            // (a block that no row of the call sees is still visited once: its old weights fade)
            if (lo < hi || (t0 == q.n_tiles && !last)) return true;
        }
        return false;
    }
};

struct WeighTcPlan {
    int64_t scan[32], targets[2];
    WeighTcSpot spot[2];
};

__device__ inline void weigh_tc_stretch(const WeighArgs& a, int TPT, WeighTcPlan& p, double inv_grid, int* status) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int WARPS = blockDim.x >> 5;
    if (threadIdx.x < 2) { p.targets[threadIdx.x] = -1; p.spot[threadIdx.x] = WeighTcSpot{a.c.batch, 0, 0, 0}; }
    const int per = (a.c.batch + (int)blockDim.x - 1) / (int)blockDim.x;
    const int lo = min((int)threadIdx.x * per, a.c.batch), hi = min(lo + per, a.c.batch);
    auto units = [&](int s) {
        const WeighTcSeq q = weigh_tc_seq(a, TPT, s);
        return (int64_t)a.c.H_kv * weigh_tc_before(q, TPT, q.n_kb);
    };
    int64_t mine = 0;
    for (int s = lo; s < hi; ++s) {
        mine += units(s);
        if (blockIdx.x == 0 && (a.c.kv_lens[s] < 0 || a.c.kv_lens[s] > paged_places(a.c)))
            report_async(status, kAsyncBadIndex, 0x801);
    }
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t below = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += below;
    }
    if (lane == 31) p.scan[warp] = upto;
    __syncthreads();
    int64_t total = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) upto += p.scan[w];
        total += p.scan[w];
    }
    for (int e = 0; e < 2; ++e) {
        int64_t u = (int64_t)((double)total * (double)(blockIdx.x + e) * inv_grid);
        if (blockIdx.x + e >= gridDim.x || u < upto - mine || u >= upto) continue;  // (one thread)
        u -= upto - mine;
        for (int s = lo; s < hi; ++s) {
            const int64_t all = units(s);
            if (u < all) {
                p.targets[e] = u;
                p.spot[e].seq = s;
                break;
            }
            u -= all;
        }
    }
    __syncthreads();
    if (lane == 0 && warp < 2 && p.targets[warp] >= 0) {
        WeighTcSpot& spot = p.spot[warp];
        const WeighTcSeq q = weigh_tc_seq(a, TPT, spot.seq);
        const int64_t per_head = weigh_tc_before(q, TPT, q.n_kb);
        int64_t u = p.targets[warp];
        spot.head = (int)(u / per_head);
        u -= spot.head * per_head;
        int b = 0, e = q.n_kb;  // before(b) <= u < before(e)
        while (e - b > 1) {
            const int mid = (b + e) >> 1;
            if (weigh_tc_before(q, TPT, mid) <= u) b = mid; else e = mid;
        }
        spot.kb = b;
        // (a boundary in the block's cost is its end)
        spot.tile = (int)min((int64_t)weigh_tc_first(q, TPT, b) + u - weigh_tc_before(q, TPT, b), (int64_t)q.n_tiles);
    }
}

// What weigh_merge_kernel has to know about a CTA: first 0 no part; 1 its first block came from an earlier CTA and goes on in a
// later one; 2 came from an earlier one and ends here; 3 begins here.  open: its last block begins here and ends later.  failed: a
// wait ran out, so that its sums may lack something and its parts are not all there.
struct WeighEnds { int first, open, seq, head, kb, failed, pad[2]; };
static_assert(sizeof(WeighEnds) == 32, "two int4");

struct WeighTcSmem {
    alignas(1024) uint8_t k[2][2][128 * 256];  // [buffer][128 keys]: [8 keys][d half][key][64 bf16], 128-byte swizzle
    alignas(1024) uint8_t q[kWtStages][128 * 256];  // [d half][row][64 bf16]
    float nl[kWtStages][128];                  // -lse of the tile's rows, base two
    alignas(16) uint32_t live[kWtStages][4];   // a bit for each row: clear where it gives nothing, whatever it holds (lse -infinity)
    union {
        float join[kWtKeys];                   // the second half of the columns' sums on their way to the first's threads
        WeighTcPlan plan;
    };
    alignas(8) uint64_t q_full[kWtStages], q_empty[kWtStages], l_full[kWtStages], l_empty[kWtStages];
    uint64_t d_full[2][2], d_empty[2][2], k_full[2], k_empty[2], k_land[2], j_full[2], j_empty[2], drain;
    uint32_t tmem_base;
    int abort;
};
static_assert(sizeof(WeighTcSmem) <= 227 * 1024, "a CTA's shared memory");

// Clamps that let a NaN through.
__device__ __forceinline__ float clamp_nan(float x, float lo, float hi) {
    float d;
    asm("{\n\t.reg .f32 a;\n\tmax.NaN.f32 a, %1, %2;\n\tmin.NaN.f32 %0, a, %3;\n\t}" : "=f"(d) : "f"(x), "f"(lo), "f"(hi));
    return d;
}

// 2^x by arithmetic, two at a time: x = n + f with n the nearest whole number, |f| <= 1/2; 2^f = 1 + f r(f) with r of degree 4
// fitted to the least relative error (1.6e-7 with fp32 roundings); twice that times 2^(n-1), a product, so that a NaN stays one (n
// added in the exponent's place would make a number of it).  From 128 on infinity; below -125.5, where 2^(n-1) is no normal
// number, zero.
__device__ __forceinline__ float2 exp2_by_arithmetic(float2 x) {
    constexpr float M = 12582912.f;  // 1.5 * 2^23: a sum with it has the whole number in its last bits
    x.x = clamp_nan(x.x, -126.f, 128.f);
    x.y = clamp_nan(x.y, -126.f, 128.f);
    const float2 t = __fadd2_rn(x, make_float2(M, M));
    const float2 n = __fadd2_rn(t, make_float2(-M, -M));
    const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
    auto both = [](float c) { return make_float2(2.f * c, 2.f * c); };
    float2 r = __ffma2_rn(both(1.326466561295092e-3f), f, both(9.671512991189957e-3f));
    r = __ffma2_rn(r, f, both(5.550733953714371e-2f));
    r = __ffma2_rn(r, f, both(0.24022242426872253f));
    r = __ffma2_rn(r, f, both(0.6931470036506653f));
    r = __ffma2_rn(r, f, both(1.f));
    return __fmul2_rn(r, make_float2(__int_as_float((__float_as_int(t.x) << 23) + 0x3F000000), __int_as_float((__float_as_int(t.y) << 23) + 0x3F000000)));
}

// n bits from bit `first` on, as far as 32 bits go.
__device__ __forceinline__ uint32_t bits_from(uint32_t first, uint32_t n) {
    uint32_t m;
    asm("bmsk.clamp.b32 %0, %1, %2;" : "=r"(m) : "r"(first), "r"(n));
    return m;
}

// Waits for this thread's loads from tensor memory; the registers are named so that nothing reads them earlier.
__device__ __forceinline__ void tmem_landed(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}

// One of eight pairs of columns takes its exponentials by arithmetic (4096 tokens on 28K: none 2.42 ms, one 2.38, two 2.43, three
// 2.55: the exponential unit is relieved, but arithmetic costs issue slots and power).
__host__ __device__ constexpr bool weigh_by_arithmetic(int pair) { return pair % 8 == 0; }
template <bool V> struct Flag { static constexpr bool value = V; };

// Warps: 0-15 sums (quadrant of lanes w mod 4, key tile (w / 4) mod 2, half of the columns w / 8), 16 issues the products, 17
// loads queries, 18 their lse, 19 loads keys, 20-23 (fp8 caches) widen them to bf16.
template <bool F8>
__global__ void __launch_bounds__(weigh_tc_threads(F8), 1)
weigh_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const WeighArgs a, int TPT, int box_keys,
                float* part, WeighEnds* ends, double inv_grid, int* status) {
    extern __shared__ __align__(1024) uint8_t weigh_smem[];  // (no room to round the base up)
    WeighTcSmem& sm = *reinterpret_cast<WeighTcSmem*>(weigh_smem);
    if ((smem_u32(weigh_smem) & 1023) != 0) {  // swizzled tiles need it; the same for every thread
        if (threadIdx.x == 0) {
            report_async(status, kAsyncBadIndex, 0x8FF);
            ends[blockIdx.x] = WeighEnds{0, 0, 0, 0, 0, 1, {}};
        }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort = &sm.abort;
    weigh_tc_stretch(a, TPT, sm.plan, inv_grid, status);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWtStages; ++i) {
            mbar_init(&sm.q_full[i], 1); mbar_init(&sm.q_empty[i], 1); mbar_init(&sm.l_full[i], 32); mbar_init(&sm.l_empty[i], kWtEpiWarps);
        }
        for (int i = 0; i < 2; ++i) {
            for (int j = 0; j < 2; ++j) { mbar_init(&sm.d_full[i][j], 1); mbar_init(&sm.d_empty[i][j], kWtEpiWarps / 2); }
            mbar_init(&sm.k_full[i], F8 ? kWtWidenWarps : 1); mbar_init(&sm.k_empty[i], 1); mbar_init(&sm.k_land[i], 1);
            mbar_init(&sm.j_full[i], kWtEpiWarps / 4); mbar_init(&sm.j_empty[i], kWtEpiWarps / 4);
        }
        mbar_init(&sm.drain, 1);
        sm.abort = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_q);
        tma_prefetch_desc(&tm_k);
    }
    if (warp == 16) tmem_alloc(&sm.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    WeighTcWalk walk(sm.plan.spot[0], sm.plan.spot[1]);
    __syncthreads();  // (the plan's memory is the sums' from here on)
    WeighPart p{};
    const int H_q = a.c.H_kv * a.G;
    bool ok = true;
    int T = 0;  // tiles so far

    if (warp < kWtEpiWarps) {
        // ---------------- sums
        const int quad = warp & 3, dd = (warp >> 2) & 1, half = warp >> 3;
        const int in_block = dd * 128 + quad * 32 + lane;
        WeighEnds e{};
        for (int n = 0; ok && walk.next(a, TPT, p); ++n) {
            const int key = p.kb * kWtKeys + in_block;
            const int first_tok = key - p.base;  // first token that sees the key
            // where the sum goes, and what stands there: looked up while the first products are made
            int64_t w = -1;
            float old = 0.f;
            if (half == 0 && p.whole() && key < p.kv) {
                const WeighPlace place = weigh_place(a, p.seq, p.head, key, status);
                if (place.row >= 0) {
                    w = place.w;
                    old = weigh_old(a, w, key, p.base);
                }
            }
            float total = 0.f;
            // Sixteen columns at a time: the next ones (the next tile's, in the end) are on their way while these are added.
            uint32_t v[2][16];
            const uint32_t lane0 = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(dd * 128 + half * 64);
            auto tile_there = [&](int tile) {
                ok = mbar_wait(&sm.d_full[tile & 1][dd], (tile >> 1) & 1, abort);
                tc_fence_after();
                return ok;
            };
            if (p.lo < p.hi && tile_there(T)) {
                tmem_ld_32x16(lane0 + (T & 1) * 256, v[0]);
                tmem_landed(v[0]);
            }
            for (int t = p.lo; ok && t < p.hi; ++t, ++T) {
                const int st = T % kWtStages, buf = T & 1;
                if (!mbar_wait(&sm.l_full[st], (T / kWtStages) & 1, abort)) { ok = false; break; }
                // visible columns [c_lo, c_hi) of this thread's key; all of them for all keys of the warp, and no row that gives
                // nothing: no masks
                const uint2 live = *reinterpret_cast<const uint2*>(&sm.live[st][half * 2]);
                const int tok0 = t * TPT;
                const int c_hi = min(TPT, p.q_len - tok0) * a.G - half * 64;
                const int c_lo = min(max(first_tok - tok0, 0), 256) * a.G - half * 64;
                const bool all = c_hi >= 64 && (live.x & live.y) == 0xFFFFFFFFu && __all_sync(0xffffffffu, c_lo <= 0);
                const float* nl = sm.nl[st] + half * 64;
                float2 s2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                auto add = [&](auto masked) {  // (two loops: with the masks in one the selects bound it)
                    uint32_t seen[2];  // a bit for each column
                    for (int w = 0; w < 2; ++w) {
                        const int lo = max(c_lo - 32 * w, 0);
                        seen[w] = (w == 0 ? live.x : live.y) & bits_from(lo, max(c_hi - 32 * w - lo, 0));
                    }
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        const bool more = ch < 3 || t + 1 < p.hi;
                        if (ch < 3) tmem_ld_32x16(lane0 + buf * 256 + (ch + 1) * 16, v[(ch + 1) & 1]);
                        else if (more && tile_there(T + 1)) tmem_ld_32x16(lane0 + (buf ^ 1) * 256, v[0]);
                        if (!decltype(masked)::value || ch * 16 < c_hi)
#pragma unroll
                        for (int c = 0; c < 16; c += 4) {
                            const float4 l = *reinterpret_cast<const float4*>(nl + ch * 16 + c);
                            const float2 sc = make_float2(a.scale_log2e, a.scale_log2e);
                            const uint32_t* w = v[ch & 1] + c;
                            float2 x[2] = {__ffma2_rn(make_float2(__uint_as_float(w[0]), __uint_as_float(w[1])), sc, make_float2(l.x, l.y)),
                                           __ffma2_rn(make_float2(__uint_as_float(w[2]), __uint_as_float(w[3])), sc, make_float2(l.z, l.w))};
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                if (weigh_by_arithmetic((c >> 1) + i)) x[i] = exp2_by_arithmetic(x[i]);
                                else { x[i].x = ex2_approx(x[i].x); x[i].y = ex2_approx(x[i].y); }
                                if constexpr (decltype(masked)::value) {
                                    const int col = ch * 16 + c + 2 * i;
                                    x[i].x = (seen[col >> 5] & 1u << (col & 31)) != 0 ? x[i].x : 0.f;
                                    x[i].y = (seen[col >> 5] & 2u << (col & 31)) != 0 ? x[i].y : 0.f;
                                }
                                s2[i] = __fadd2_rn(s2[i], x[i]);
                            }
                        }
                        if (more) tmem_landed(v[(ch + 1) & 1]);
                        if (ch == 2) {  // the tile is in registers
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&sm.d_empty[buf][dd]);
                        }
                    }
                };
                if (all) add(Flag<false>{});
                else add(Flag<true>{});
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.l_empty[st]);
                total += (s2[0].x + s2[0].y) + (s2[1].x + s2[1].y);
            }
            if (!ok && lane == 0) report_async(status, kAsyncTimeout, 0x821);
            // the two halves of the columns, then the key's place (or this CTA's partial sums)
            if (half == 1) {
                ok = ok && (n == 0 || mbar_wait(&sm.j_empty[dd], (n - 1) & 1, abort));
                if (ok) sm.join[in_block] = total;  // (else the sums before it may still be read)
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.j_full[dd]);
            } else {
                ok = ok && mbar_wait(&sm.j_full[dd], n & 1, abort);
                // (the other half's wait may have run out where this one's has not: it says so before it hands over its sum)
                const int gone = *abort;
                total += sm.join[in_block];
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.j_empty[dd]);
                const int which = p.lo > p.t0 ? 0 : 1;
                ok = ok && gone == 0;
                if (!ok) {
                    // what stands in the pool stays: it is the sum of many steps
                } else if (p.whole()) {
                    if (w >= 0) a.w[w] = old + total;
                } else {
                    part[((int64_t)blockIdx.x * 2 + which) * kWtKeys + in_block] = total;
                }
            }
            if (e.first == 0) e.first = p.lo == p.t0 ? 3 : (p.hi < p.n ? 1 : 2);
            e.open = p.lo == p.t0 && p.hi < p.n;
            e.seq = p.seq; e.head = p.head; e.kb = p.kb;
        }
        if (threadIdx.x == 0) ends[blockIdx.x] = e;
    } else if (warp == 16) {
        // ---------------- products
        constexpr uint32_t idesc = make_idesc_bf16(128, 128, false, false);
        for (int i = 0; ok && walk.next(a, TPT, p); ++i) {
            const int kb = i & 1;
            if (!mbar_wait(&sm.k_full[kb], (i >> 1) & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x822);
                break;
            }
            for (int t = p.lo; t < p.hi; ++t, ++T) {
                const int st = T % kWtStages, buf = T & 1;
                ok = mbar_wait(&sm.q_full[st], (T / kWtStages) & 1, abort);
                for (int dd = 0; ok && dd < 2; ++dd) {
                    if (T > 1) ok = mbar_wait(&sm.d_empty[buf][dd], ((T >> 1) - 1) & 1, abort);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t kd = make_smem_desc(smem_u32(sm.k[kb][dd]), 16, 2048), qd = make_smem_desc(smem_u32(sm.q[st]), 16, 1024);
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)  // 16 of d: 32 bytes of a row; the second 64 are 1 KB on, of the queries 16 KB
                            mma_bf16_ss(tmem + (buf * 2 + dd) * 128, kd + (uint64_t)((kk >> 2) * 64 + 2 * (kk & 3)),
                                        qd + (uint64_t)((kk >> 2) * 1024 + 2 * (kk & 3)), idesc, kk > 0);
                        mma_commit(&sm.d_full[buf][dd]);
                        if (dd == 1) mma_commit(&sm.q_empty[st]);
                        if (dd == 1 && t == p.hi - 1) mma_commit(&sm.k_empty[kb]);
                    }
                    __syncwarp();
                }
                if (!ok) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x823);
                    break;
                }
            }
            if (p.lo >= p.hi && lane == 0) mbar_arrive(&sm.k_empty[kb]);  // (nothing to multiply)
        }
    } else if (warp == 17) {
        // ---------------- queries: two boxes (halves of d) of TPT tokens' heads of the group
        if (const long long late = g_debug_producer_delay; late > 0) spin_cycles(late);  // tests only
        const uint32_t bytes = (uint32_t)(TPT * a.G) * 256;
        while (ok && walk.next(a, TPT, p)) {
            for (int t = p.lo; t < p.hi; ++t, ++T) {
                const int st = T % kWtStages;
                if (T >= kWtStages && !mbar_wait(&sm.q_empty[st], (T / kWtStages - 1) & 1, abort)) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x824);
                    ok = false;
                    break;
                }
                if (lane == 0) {
                    mbar_arrive_expect_tx(&sm.q_full[st], bytes);
                    for (int h = 0; h < 2; ++h) tma_load_3d(sm.q[st] + h * 16384, &tm_q, h * 64, p.head * a.G, p.q_row + t * TPT, &sm.q_full[st]);
                }
                __syncwarp();
            }
        }
    } else if (warp == 18) {
        // ---------------- lse of the rows, four a lane, a tile ahead; which of them give nothing
        int tok[4], at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 32 + lane;
            tok[i] = r < TPT * a.G ? r / a.G : 1 << 30;
            at[i] = r / a.G * H_q + r % a.G;
        }
        while (ok && walk.next(a, TPT, p)) {
            const float* lse = a.lse + (int64_t)p.q_row * H_q + p.head * a.G;
            float l[4], ahead[4];
            auto fetch = [&](int t, float (&x)[4]) {
                const float* from = lse + (int64_t)t * TPT * H_q;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = t < p.hi && tok[i] < p.q_len - t * TPT ? __ldg(from + at[i]) : 0.f;
            };
            fetch(p.lo, ahead);
            for (int t = p.lo; t < p.hi; ++t, ++T) {
                const int st = T % kWtStages;
#pragma unroll
                for (int i = 0; i < 4; ++i) l[i] = ahead[i];
                fetch(t + 1, ahead);
                if (T >= kWtStages && !__all_sync(0xffffffffu, mbar_wait(&sm.l_empty[st], (T / kWtStages - 1) & 1, abort))) {
                    if (lane == 0) report_async(status, kAsyncTimeout, 0x826);
                    ok = false;
                    break;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool out = l[i] == -INFINITY;
                    const uint32_t live = ~__ballot_sync(0xffffffffu, out);
                    if (lane == 0) sm.live[st][i] = live;
                    sm.nl[st][i * 32 + lane] = out ? -INFINITY : -l[i] * 1.4426950408889634f;
                }
                mbar_arrive(&sm.l_full[st]);
            }
        }
    } else if (warp == 19) {
        // ---------------- keys: one box per page (or 128 keys of a larger one), a lane each, two blocks on their way
        const int boxes = kWtKeys / box_keys;
        const int nowhere = F8 ? a.c.n_pages * a.c.page_size : a.c.n_pages * a.c.page_size / 8;  // reads as zeros
        auto place_of = [&]() {
            const uint32_t key = (uint32_t)p.kb * kWtKeys + lane * box_keys, size = a.c.page_size;  // (below 2^31 + 256)
            if (lane >= boxes || key >= (uint32_t)p.kv) return nowhere;
            const uint32_t slot = key / size;
            const int page = a.c.table[(int64_t)p.seq * a.c.max_pages + slot];
            if (page < 0 || page >= a.c.n_pages) {
                report_async(status, kAsyncBadIndex, 0x802);
                return nowhere;
            }
            const int row = page * a.c.page_size + (int)(key - slot * size);
            return F8 ? row : row / 8;
        };
        for (int i = 0; walk.next(a, TPT, p); ++i) {
            const int where = place_of(), buf = i & 1;
            if (i >= 2 && !mbar_wait(&sm.k_empty[buf], ((i >> 1) - 1) & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x825);
                break;
            }
            uint64_t* bar = F8 ? &sm.k_land[buf] : &sm.k_full[buf];
            if (lane == 0) mbar_arrive_expect_tx(bar, kWtKeys * (F8 ? 128 : 256));
            __syncwarp();
            uint8_t* dst = sm.k[buf][0];
            if (lane < boxes) {
                // (fp8: 32 keys into the upper half of the 8 KB of their bf16)
                if constexpr (F8) tma_load_3d(dst + (lane * box_keys >> 5) * 8192 + 4096 + (lane * box_keys & 31) * 128, &tm_k, 0, p.head, where, bar);
                else tma_load_5d(dst + lane * box_keys * 256, &tm_k, 0, 0, 0, p.head, where, bar);
            }
            __syncwarp();
        }
    } else if constexpr (F8) {
        // ---------------- widening: 64 keys of a block a warp, 32 at a time
        const int w = warp - 20;
        for (int i = 0; walk.next(a, TPT, p); ++i) {
            const int buf = i & 1;
            if (!mbar_wait(&sm.k_land[buf], (i >> 1) & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x827);
                break;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint8_t* keys = sm.k[buf][0] + (w * 2 + h) * 8192;
                uint4 x[8];
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const int k = s * 4 + (lane >> 3), chunk = lane & 7;
                    x[s] = *reinterpret_cast<const uint4*>(keys + 4096 + k * 128 + ((chunk ^ (k & 7)) << 4));
                }
                __syncwarp();
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const int k = s * 4 + (lane >> 3), chunk = lane & 7;
                    const uint32_t v[4] = {x[s].x, x[s].y, x[s].z, x[s].w};
                    uint32_t o[8];
                    e4m3x16_to_bf16x16(v, o);
                    uint8_t* to = keys + (k >> 3) * 2048 + (chunk >> 2) * 1024 + (k & 7) * 128;
                    *reinterpret_cast<uint4*>(to + (((2 * chunk & 7) ^ (k & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(to + ((((2 * chunk + 1) & 7) ^ (k & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
            fence_proxy_async_smem();  // written through the generic proxy, read by the products
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.k_full[buf]);
        }
    }
    if (*abort != 0) spin_cycles(200000);  // copies in flight land
    __syncwarp();
    if (warp == 16) {  // products in flight end before their memory goes
        if (elect_one()) mma_commit(&sm.drain);
        __syncwarp();
        mbar_wait_quiet(&sm.drain, 0, 20000000);
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort != 0) ends[blockIdx.x].failed = 1;
    if (warp == 16) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Adds up the key blocks that the boundaries between CTAs cut: CTA c the one that c begins and a later one ends.
__global__ void __launch_bounds__(kWtKeys)
weigh_merge_kernel(const WeighArgs a, int TPT, const float* part, const WeighEnds* ends, int n_ctas, int* status) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = blockIdx.x;
    const WeighEnds e = ends[c];
    if (e.open == 0 || e.failed != 0) return;
    float sum = part[((int64_t)c * 2 + 1) * kWtKeys + threadIdx.x];
    for (int i = c + 1; i < n_ctas; ++i) {
        const int first = ends[i].first;
        if (ends[i].failed != 0) return;
        if (first == 3) break;
        if (first == 0) continue;
        sum += part[(int64_t)i * 2 * kWtKeys + threadIdx.x];
        if (first == 2) break;
    }
    const WeighTcSeq q = weigh_tc_seq(a, TPT, e.seq);
    const int64_t key = (int64_t)e.kb * kWtKeys + threadIdx.x;
    if (key >= q.kv) return;
    const WeighPlace w = weigh_place(a, e.seq, e.head, (int)key, status);
    if (w.row >= 0) a.w[w.w] = weigh_old(a, w.w, (int)key, q.base) + sum;
}

}  // namespace msa
