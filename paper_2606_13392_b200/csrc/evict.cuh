// Keeping a paged cache within a budget (include/msa.h: msa_paged_keep, msa_paged_compact): which tokens of a sequence stay,
// for each KV head, and their move to the front of the sequence's pages.
#pragma once

#include <cooperative_groups.h>

#include "norm_rope.cuh"
#include "order.cuh"

namespace msa {

// ---------------------------------------------------------------- which tokens stay
// The middle of a sequence (between its first `sinks` and its last `recent` tokens) keeps the `need` largest weights, ties
// to the lower place.  A cluster of CTAs per (sequence, head), each with a run of the middle whose keys it holds in shared memory,
// finds the need-th largest by its bits, 11, 11 and 10 at a time: a count of the values of each digit, then the digit in which the
// need-th falls.  Two more passes count and write the places in order: a warp owns a run, so only totals are exchanged.
struct KeepArgs {
    PagedView c;
    const float* w;     // [n_pages, H_kv, page_size]
    int32_t* keep;      // [batch, H_kv, budget]
    int32_t* new_lens;  // [batch] or null
    int budget, sinks, recent;
    int cached;         // keys of a CTA that fit its shared memory (beyond, weights are read again)
};

constexpr int kKeepThreads = 1024, kKeepWarps = 32, kKeepBins = 2048, kKeepCtas = 8;

struct KeepSmem {
    uint32_t hist[3][kKeepBins];
    uint32_t scan[33], found[2];
    uint2 totals[kKeepCtas];  // above, equal: of every CTA
    alignas(16) uint32_t key[1];
};

// VEC: weights that a lane reads at a time, 4 where pages are whole runs of 16 bytes.
template <int VEC>
__global__ void __launch_bounds__(kKeepThreads)
paged_keep_kernel(const KeepArgs a, int* status) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint8_t keep_smem[];
    KeepSmem& sm = *reinterpret_cast<KeepSmem*>(keep_smem);
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int unit = blockIdx.x / ctas, s = unit / a.c.H_kv, head = unit - s * a.c.H_kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t cap = (int64_t)a.c.max_pages * a.c.page_size;
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
    // keys of places at .. at + VEC - 1
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
        for (int e = 0; e < VEC; ++e) key[e] = order_key(v[e]);
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
        auto count = [&](int at, const uint32_t (&key)[VEC]) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (at + e >= lo && at + e < hi && (round == 0 || key[e] >> (shift + bits) == prefix))
                    atomicAdd(&hist[(key[e] >> shift) & ((1u << bits) - 1)], 1u);
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
                    count(at, key[u]);
                }
            }
        } else {
            for (int at = run_lo + lane * VEC; at < run_hi; at += 32 * VEC) {
                uint32_t key[VEC];
                keys_at(at, key);
                count(at, key);
            }
        }
        if (ctas > 1) cluster.sync();
        else __syncthreads();
        // digits from the top: two a thread
        const int d = kKeepBins - 1 - 2 * (int)threadIdx.x;
        uint32_t c0 = 0, c1 = 0;
        for (int c = 0; c < ctas; ++c) {
            const uint2 x = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(hist + d - 1, c));
            c0 += x.y;
            c1 += x.x;
        }
        uint32_t all;
        const uint32_t above = block_scan(c0 + c1, sm.scan, &all);
        if (above < want && above + c0 + c1 >= want) {  // (one thread)
            const bool first = above + c0 >= want;
            sm.found[0] = first ? d : d - 1;
            sm.found[1] = want - above - (first ? 0u : c0);
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
            const bool in = at + e >= lo && at + e < hi;
            mine_above += in && key[e] > prefix;
            mine_equal += in && key[e] == prefix;
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
            const bool in = at + e >= lo && at + e < hi;
            eq += in && key[e] == prefix;
            ab += in && key[e] > prefix;
        }
        if (!__any_sync(0xffffffffu, (eq | ab) != 0)) continue;
        uint32_t both = eq << 16 | ab, upto = both;  // (at most 128 each)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t below = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += below;
        }
        uint32_t order = equal + (upto - both >> 16), above = rank_above + (upto - both & 0xFFFFu);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool in = at + e >= lo && at + e < hi, same = in && key[e] == prefix, more = in && key[e] > prefix;
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
struct CompactArgs {
    PagedView c;
    uint8_t* pool[2];     // keys and values; a null one is not moved
    float* w;             // or null
    const int32_t* keep;  // [batch, H_kv, width]
    int width, row_bytes, slice_bytes;
};

constexpr int kCompactThreads = 256, kCompactLoads = 4;

// Row of a pool that a place stands at, -1: nowhere.
__device__ __forceinline__ int64_t compact_row(const PagedView& c, const int32_t* table, int place, int64_t len, int* status) {
    if (place < 0) return -1;
    if (place >= len) {
        report_async(status, kAsyncBadIndex, 0xA01);
        return -1;
    }
    const int page = table[(uint32_t)place / (uint32_t)c.page_size];
    if (page < 0 || page >= c.n_pages) {
        report_async(status, kAsyncBadIndex, 0xA02);
        return -1;
    }
    return (int64_t)page * c.page_size + (uint32_t)place % (uint32_t)c.page_size;
}

// V: what a lane moves at a time.  blockIdx.y: slice of the keys, of the values, then the weights.
// A run of rows is looked up (a thread a row, to shared memory) while the one before it is read, and read while the one before
// that is written: its sources lie behind everything that is written then.
template <class V>
__global__ void __launch_bounds__(kCompactThreads)
paged_compact_kernel(const CompactArgs a, int slices, int* status) {
    __shared__ int64_t s_from[3][kCompactThreads], s_to[3][kCompactThreads];
    const int s = blockIdx.x / a.c.H_kv, head = blockIdx.x - s * a.c.H_kv;
    const int32_t* keep = a.keep + (int64_t)blockIdx.x * a.width;
    const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
    const int64_t len = min((int64_t)max(a.c.kv_lens[s], 0), (int64_t)a.c.max_pages * a.c.page_size);
    const int part = blockIdx.y;
    // source and destination of the i-th token, -1: it does not move
    auto look_up = [&](int i, int64_t& from, int64_t& to) {
        const int place = i < a.width ? keep[i] : -1;
        if (place >= 0 && place < i) report_async(status, kAsyncBadIndex, 0xA03);  // (not ascending from 0)
        to = -1;
        if (place <= i) return;
        from = compact_row(a.c, table, place, len, status);
        to = from >= 0 ? compact_row(a.c, table, i, len, status) : -1;
    };
    if (part == 2 * slices) {
        for (int first = 0; first < a.width; first += kCompactThreads * kCompactLoads) {
            float v[kCompactLoads];
            int64_t to[kCompactLoads];
#pragma unroll
            for (int j = 0; j < kCompactLoads; ++j) {
                int64_t row;
                look_up(first + j * kCompactThreads + (int)threadIdx.x, row, to[j]);
                if (to[j] >= 0) {
                    const int64_t off = row % a.c.page_size, off2 = to[j] % a.c.page_size;
                    v[j] = a.w[(row - off) * a.c.H_kv + (int64_t)head * a.c.page_size + off];
                    to[j] = (to[j] - off2) * a.c.H_kv + (int64_t)head * a.c.page_size + off2;
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kCompactLoads; ++j)
                if (to[j] >= 0) a.w[to[j]] = v[j];
            __syncthreads();
        }
        return;
    }
    uint8_t* pool = a.pool[part >= slices];
    if (pool == nullptr) return;
    const int slice = part >= slices ? part - slices : part;
    const int lanes = a.slice_bytes / (int)sizeof(V), rows = kCompactThreads / lanes;  // rows of a load of the CTA
    const int in_row = threadIdx.x % lanes, row0 = threadIdx.x / lanes;
    const int64_t column = (int64_t)head * a.row_bytes + slice * a.slice_bytes + in_row * (int)sizeof(V);
    const int64_t pitch = (int64_t)a.c.H_kv * a.row_bytes;
    const int run = min(rows * kCompactLoads, kCompactThreads), runs = (a.width + run - 1) / run;
    auto prepare = [&](int r) {  // run r's rows
        if ((int)threadIdx.x >= run) return;
        int64_t from = 0, to = -1;
        if (r < runs) look_up(r * run + (int)threadIdx.x, from, to);
        s_from[r % 3][threadIdx.x] = from;
        s_to[r % 3][threadIdx.x] = to;
    };
    auto read = [&](int r, V (&v)[kCompactLoads]) {
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j) {
            const int i = j * rows + row0;
            if (row0 < rows && i < run && s_to[r % 3][i] >= 0) v[j] = *reinterpret_cast<const V*>(pool + s_from[r % 3][i] * pitch + column);
        }
    };
    auto write = [&](int r, const V (&v)[kCompactLoads]) {
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j) {
            const int i = j * rows + row0;
            if (row0 < rows && i < run && s_to[r % 3][i] >= 0) *reinterpret_cast<V*>(pool + s_to[r % 3][i] * pitch + column) = v[j];
        }
    };
    V v[2][kCompactLoads];
    prepare(0);
    prepare(1);
    __syncthreads();
    read(0, v[0]);
    for (int r = 0; r < runs; r += 2) {  // (two runs' registers, taken in turn)
        read(r + 1, v[1]);       // (nothing beyond the last run: its rows say so)
        prepare(r + 2);
        __syncthreads();         // all of run r has been read
        write(r, v[0]);
        if (r + 1 >= runs) break;
        __syncthreads();         // the rows of run r + 2 are there; those of run r are not needed any more
        read(r + 2, v[0]);
        prepare(r + 3);
        __syncthreads();
        write(r + 1, v[1]);
        __syncthreads();
    }
}

}  // namespace msa
