// Keeping a paged cache within a budget (include/msa.h: msa_paged_keep, msa_paged_compact): which tokens of a sequence stay,
// for each KV head, and their move to the front of the sequence's pages.
#pragma once

#include <cooperative_groups.h>

#include "norm_rope.cuh"
#include "order.cuh"
#include "weigh.cuh"

namespace msa {

// ---------------------------------------------------------------- which tokens stay
// The middle of a sequence (between its first `sinks` and its last `recent` tokens) keeps the `need` largest weights, ties
// to the lower place.  A cluster of CTAs per (sequence, head), each with a run of the middle whose keys it holds in shared memory,
// finds the need-th largest by its bits, 11, 11 and 10 at a time: a count of the values of each digit, then the digit in which the
// need-th falls.  Two more passes count and write the places in order: a warp owns a run, so only totals are exchanged.
// Measured (8 heads): 4160 tokens of 32 sequences to 4096 13 - 15 us, bound by the rounds' latencies (some 1.5 us each of ten); 60000 -
// 262144 of 3 prompts to 2048 38 - 44 us, a million of one to 4096 130 us (five passes over what a CTA holds, instructions).
struct KeepArgs {
    PagedView c;
    const float* w;     // [n_pages, H_kv, page_size]
    int32_t* keep;      // [batch, H_kv, budget]
    int32_t* new_lens;  // [batch] or null
    int budget, sinks, recent;
    int cached;         // keys of a CTA that fit its shared memory (beyond, weights are read again)
};

constexpr int kKeepBins = 2048, kKeepCtas = 8;

struct KeepSmem {
    alignas(16) uint32_t hist[3][kKeepBins];
    uint32_t scan[33], found[2];
    uint2 totals[kKeepCtas];  // above, equal: of every CTA
    alignas(16) uint32_t key[4];
};

// VEC: weights that a lane reads at a time, 4 where pages are whole runs of 16 bytes.
template <int VEC, int kKeepThreads>
__global__ void __launch_bounds__(kKeepThreads, 1024 / kKeepThreads)
paged_keep_kernel(const KeepArgs a, int* status) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint8_t keep_smem[];
    KeepSmem& sm = *reinterpret_cast<KeepSmem*>(keep_smem);
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int unit = blockIdx.x / ctas, s = unit / a.c.H_kv, head = unit - s * a.c.H_kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kKeepWarps = kKeepThreads / 32;
    const int64_t cap = paged_places(a.c);
    const int len = a.c.kv_lens[s];
    if ((len < 0 || len > cap) && threadIdx.x == 0 && head == 0 && rank == 0) report_async(status, kAsyncBadIndex, 0x901);
    const int L = (int)min((int64_t)max(len, 0), cap);
    const int n = min(L, a.budget), recent = min(a.recent, n), sinks = min(a.sinks, n - recent);
    const int lo = sinks, hi = L - recent, need = n - recent - sinks;  // the middle [lo, hi) keeps `need`
    int32_t* out = a.keep + (int64_t)unit * a.budget;
    if (a.new_lens != nullptr && threadIdx.x == 0 && head == 0 && rank == 0) a.new_lens[s] = n;
    for (int i = rank * kKeepThreads + threadIdx.x; i < a.budget; i += ctas * kKeepThreads) {
        if (i < sinks || (L == n && i < n)) out[i] = i;
        else if (i >= n) out[i] = -1;
        else if (i >= n - recent) out[i] = L - n + i;
    }
    if (L == n || need == 0) return;

    for (int i = threadIdx.x; i < 3 * kKeepBins; i += kKeepThreads) sm.hist[0][i] = 0;
    const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
    const uint32_t size = a.c.page_size;
    // a warp's run of places, in steps of 32 VEC from a multiple of VEC
    const int from = lo / VEC * VEC, steps = (hi - from + 32 * VEC - 1) / (32 * VEC), per = (steps + ctas * kKeepWarps - 1) / (ctas * kKeepWarps);
    const int w0 = rank * kKeepWarps + warp;
    const int run_lo = from + min(steps, w0 * per) * 32 * VEC, run_hi = from + min(steps, (w0 + 1) * per) * 32 * VEC;
    // keys of places at .. at + VEC - 1: 0 outside the middle, where nothing else has it (a NaN has 1, -infinity more)
    auto keys_of = [&](int at, uint32_t (&key)[VEC]) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = __int_as_float(0x7fc00000);
        if (at < hi) {
            const uint32_t slot = (uint32_t)at / size;
            const int page = table[slot];
            if (page >= 0 && page < a.c.n_pages) {
                const float* x = a.w + ((int64_t)page * a.c.H_kv + head) * size + ((uint32_t)at - slot * size);
                if constexpr (VEC == 4) {
                    const float4 f = __ldg(reinterpret_cast<const float4*>(x));
                    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
                } else {
                    v[0] = __ldg(x);
                }
            } else {
                report_async(status, kAsyncBadIndex, 0x902);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) key[e] = at + e >= lo && at + e < hi ? max(order_key(v[e]), 1u) : 0u;
    };
    // ... from this warp's part of shared memory as far as that goes
    const int mine_cached = min(run_hi - run_lo, a.cached / kKeepWarps / (32 * VEC) * (32 * VEC));
    uint32_t* cache = sm.key + warp * (a.cached / kKeepWarps / (32 * VEC) * (32 * VEC));
    auto keys_at = [&](int at, uint32_t (&key)[VEC]) {
        if (at - run_lo < mine_cached) {
            if constexpr (VEC == 4) {
                const uint4 k = *reinterpret_cast<const uint4*>(cache + (at - run_lo));
                key[0] = k.x; key[1] = k.y; key[2] = k.z; key[3] = k.w;
            } else {
                key[0] = cache[at - run_lo];
            }
        } else {
            keys_of(at, key);
        }
    };
    __syncthreads();

    // ---- the need-th largest key
    uint32_t want = need, prefix = 0;
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
        uint32_t* hist = sm.hist[round];
        auto count = [&](const uint32_t (&key)[VEC]) {  // (what is outside is counted below everything: it changes nothing)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (round == 0 || key[e] >> (shift + bits) == prefix) atomicAdd(&hist[(key[e] >> shift) & ((1u << bits) - 1)], 1u);
        };
        if (round == 0) {
            constexpr int U = 4;  // pieces in flight
            for (int at0 = run_lo + lane * VEC; at0 < run_hi; at0 += U * 32 * VEC) {
                uint32_t key[U][VEC];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (at0 + u * 32 * VEC < run_hi) keys_of(at0 + u * 32 * VEC, key[u]);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int at = at0 + u * 32 * VEC;
                    if (at >= run_hi) break;
                    if (at - run_lo < mine_cached) {
                        if constexpr (VEC == 4) *reinterpret_cast<uint4*>(cache + (at - run_lo)) = make_uint4(key[u][0], key[u][1], key[u][2], key[u][3]);
                        else cache[at - run_lo] = key[u][0];
                    }
                    count(key[u]);
                }
            }
        } else {
            for (int at = run_lo + lane * VEC; at < run_hi; at += 32 * VEC) {
                uint32_t key[VEC];
                keys_at(at, key);
                count(key);
            }
        }
        if (ctas > 1) cluster.sync();
        else __syncthreads();
        // digits from the top, a few a thread
        constexpr int PER = kKeepBins / kKeepThreads;
        static_assert(PER == 2 || PER == 4, "read as one");
        const int d = kKeepBins - PER * (1 + (int)threadIdx.x);
        uint32_t c[PER] = {}, mine = 0, all;
        for (int r = 0; r < ctas; ++r) {
            if constexpr (PER == 2) {
                const uint2 x = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(hist + d, r));
                c[0] += x.x; c[1] += x.y;
            } else {
                const uint4 x = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(hist + d, r));
                c[0] += x.x; c[1] += x.y; c[2] += x.z; c[3] += x.w;
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) mine += c[j];
        uint32_t above = block_scan(mine, sm.scan, &all);
#pragma unroll
        for (int j = PER - 1; j >= 0; --j) {
            if (above < want && above + c[j] >= want) { sm.found[0] = d + j; sm.found[1] = want - above; }  // (one thread)
            above += c[j];
        }
        __syncthreads();
        prefix = round == 0 ? sm.found[0] : (prefix << bits) | sm.found[0];
        want = sm.found[1];
    }
    // ---- kept: keys above `prefix`, and the first `want` of those equal to it
    uint32_t mine_above = 0, mine_equal = 0;
    for (int at = run_lo + lane * VEC; at < run_hi; at += 32 * VEC) {
        uint32_t key[VEC];
        keys_at(at, key);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            mine_above += key[e] > prefix;
            mine_equal += key[e] == prefix;
        }
    }
    mine_above = __reduce_add_sync(0xffffffffu, mine_above);
    mine_equal = __reduce_add_sync(0xffffffffu, mine_equal);
    uint32_t cta_above, cta_equal;
    uint32_t rank_above = block_scan(lane == 0 ? mine_above : 0u, sm.scan, &cta_above);  // of earlier warps
    uint32_t equal = block_scan(lane == 0 ? mine_equal : 0u, sm.scan, &cta_equal);
    if (ctas > 1) {
        if (threadIdx.x < ctas) cluster.map_shared_rank(&sm, threadIdx.x)->totals[rank] = make_uint2(cta_above, cta_equal);
        cluster.sync();
        for (int c = 0; c < rank; ++c) {
            rank_above += sm.totals[c].x;
            equal += sm.totals[c].y;
        }
    }
    rank_above = __shfl_sync(0xffffffffu, rank_above, 0);
    equal = __shfl_sync(0xffffffffu, equal, 0);
    for (int at0 = run_lo; at0 < run_hi; at0 += 32 * VEC) {
        const int at = at0 + lane * VEC;
        uint32_t key[VEC];
        keys_at(at, key);
        uint32_t eq = 0, ab = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            eq += key[e] == prefix;
            ab += key[e] > prefix;
        }
        if (!__any_sync(0xffffffffu, eq != 0)) {  // (nearly always: who is kept is seen by all)
            uint32_t before = 0, own = 0, sum = 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const uint32_t who = __ballot_sync(0xffffffffu, key[e] > prefix);
                before += __popc(who & ((1u << lane) - 1));
                sum += __popc(who);
            }
            const uint32_t to = sinks + rank_above + min(equal, want) + before;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (key[e] > prefix) out[to + own++] = at + e;
            rank_above += sum;
            continue;
        }
        uint32_t both = eq << 16 | ab, upto = both;  // (at most 128 each)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t below = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += below;
        }
        uint32_t order = equal + (upto - both >> 16), above = rank_above + (upto - both & 0xFFFFu);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool same = key[e] == prefix, more = key[e] > prefix;
            if (more || (same && order < want)) out[sinks + above + min(order, want)] = at + e;  // (places before it that stay)
            order += same;
            above += more;
        }
        const uint32_t last = __shfl_sync(0xffffffffu, upto, 31);
        equal += last >> 16;
        rank_above += last & 0xFFFFu;
    }
}

// ---------------------------------------------------------------- their move
// Token keep[i] goes to place i of its (sequence, head): in place, so a row may only be overwritten once it has been read.
// keep is ascending: sources of a run of places lie behind the sources of the runs before and not before the run itself.
// So a CTA that goes through the places in order, reading a run before writing it, is safe - and the slices of a row are
// independent of each other, which is where the parallelism comes from: a CTA per (sequence, head, pool, slice of a row).
// Measured (8 heads of 128): 4096 of 4160 tokens of 32 sequences 203 us, 80 % of the copy bandwidth; of one sequence of 8192 18 us;
// 2048 of 30000 - 65536 of 3 prompts on fp8 21 us (bound by the chain place -> page -> row of two runs, and by launch).
struct CompactArgs {
    PagedView c;
    uint8_t* pool[2];     // keys and values; a null one is not moved
    float* w;             // or null
    const int32_t* keep;  // [batch, H_kv, width]
    int width, row_bytes, slice_bytes;
};

constexpr int kCompactLoads = 4;

// V: what a lane moves at a time.  blockIdx.y: slice of the keys, of the values; the first slice of the keys moves the weights, too.
// A run of rows (a thread looks up one) is read while the run before it is written: its sources lie behind everything that is
// written then.  The look-ups are spread over the runs before, one load of the chain place -> pages -> rows in each.
// kCompactThreads: 256, four CTAs per SM; 1024 where there are few.
template <class V, int kCompactThreads>
__global__ void __launch_bounds__(kCompactThreads, 1024 / kCompactThreads)
paged_compact_kernel(const CompactArgs a, int slices, int* status) {
    __shared__ int64_t s_from[3][kCompactThreads], s_to[3][kCompactThreads];  // rows of the pools; to = -1: it does not move
    const int s = blockIdx.x / a.c.H_kv, head = blockIdx.x - s * a.c.H_kv, tid = threadIdx.x;
    const int32_t* keep = a.keep + (int64_t)blockIdx.x * a.width;
    const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
    const int said = a.c.kv_lens[s], len = (int)min((int64_t)max(said, 0), paged_places(a.c));
    const bool values = (int)blockIdx.y >= slices, weights = blockIdx.y == 0 && a.w != nullptr;
    uint8_t* pool = a.pool[values];
    const int slice = values ? blockIdx.y - slices : blockIdx.y;
    const int lanes = a.slice_bytes / (int)sizeof(V), rows = kCompactThreads / lanes;  // rows of a load of the CTA
    const int in_row = tid % lanes, row0 = tid / lanes;
    const int64_t column = (int64_t)head * a.row_bytes + slice * a.slice_bytes + in_row * (int)sizeof(V);
    const int64_t pitch = (int64_t)a.c.H_kv * a.row_bytes;
    const int run = min(rows * kCompactLoads, kCompactThreads), runs = (a.width + run - 1) / run;
    const uint32_t size = a.c.page_size;

    // the chain of a thread's row of a run: its place; the pages of where it is and where it goes; the rows
    int place_next = -1, place = -1, page_from = -1, page_to = -1;
    auto load_place = [&](int r) {
        const int i = r * run + tid;
        place_next = tid < run && i < a.width ? keep[i] : -1;
    };
    auto load_pages = [&](int r) {
        const int i = r * run + tid;
        place = place_next;
        if (place >= 0 && place < i) report_async(status, kAsyncBadIndex, 0xA03);  // (not ascending from 0)
        // (a bad length is reported where a place beyond it would be: a branch of its own cost 4 - 12 % by the code around it)
        if (place >= len || (r == 0 && said != len)) report_async(status, kAsyncBadIndex, 0xA01);
        if (place > i && place < len) {
            page_from = table[(uint32_t)place / size];
            page_to = table[(uint32_t)i / size];
        } else {
            place = -1;  // (it does not move)
        }
    };
    auto set_rows = [&](int r) {
        const int i = r * run + tid;
        const bool moves = place >= 0, good = page_from >= 0 && page_from < a.c.n_pages && page_to >= 0 && page_to < a.c.n_pages;
        if (moves && !good) report_async(status, kAsyncBadIndex, 0xA02);
        s_from[r % 3][tid] = moves && good ? (int64_t)page_from * size + (uint32_t)place % size : 0;
        s_to[r % 3][tid] = moves && good ? (int64_t)page_to * size + (uint32_t)i % size : -1;
    };
    auto weight_at = [&](int64_t row) { return (row / size * a.c.H_kv + head) * size + row % size; };
    auto read = [&](int r, V (&v)[kCompactLoads], float& w) {
        const int64_t* from = s_from[r % 3];
        const int64_t* to = s_to[r % 3];
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j) {
            const int i = j * rows + row0;
            if (row0 < rows && i < run && to[i] >= 0 && pool != nullptr) v[j] = *reinterpret_cast<const V*>(pool + from[i] * pitch + column);
        }
        if (weights && tid < run && to[tid] >= 0) w = a.w[weight_at(from[tid])];
    };
    auto write = [&](int r, const V (&v)[kCompactLoads], float w) {
        const int64_t* to = s_to[r % 3];
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j) {
            const int i = j * rows + row0;
            if (row0 < rows && i < run && to[i] >= 0 && pool != nullptr) *reinterpret_cast<V*>(pool + to[i] * pitch + column) = v[j];
        }
        if (weights && tid < run && to[tid] >= 0) a.w[weight_at(to[tid])] = w;
    };
    V v[2][kCompactLoads];
    float w[2];
    load_place(0); load_pages(0); load_place(1); set_rows(0);
    load_pages(1); load_place(2); set_rows(1);
    load_pages(2); load_place(3);
    __syncthreads();
    read(0, v[0], w[0]);
    for (int r = 0; r < runs; r += 2) {  // (two runs' registers, taken in turn; rows beyond the last run do not move)
        read(r + 1, v[1], w[1]);
        set_rows(r + 2); load_pages(r + 3); load_place(r + 4);
        __syncthreads();  // all of run r has been read
        write(r, v[0], w[0]);
        if (r + 1 >= runs) break;
        __syncthreads();  // its rows are not needed any more
        read(r + 2, v[0], w[0]);
        set_rows(r + 3); load_pages(r + 4); load_place(r + 5);
        __syncthreads();
        write(r + 1, v[1], w[1]);
        __syncthreads();
    }
}

}  // namespace msa
