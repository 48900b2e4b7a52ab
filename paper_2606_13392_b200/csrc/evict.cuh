// Keeping a paged cache within a budget (include/msa.h: msa_paged_keep, msa_paged_compact): which tokens of a sequence stay,
// for each KV head, and their move to the front of the sequence's pages.
#pragma once

#include "norm_rope.cuh"
#include "order.cuh"

namespace msa {

// ---------------------------------------------------------------- which tokens stay
// The middle of a sequence (between its first `sinks` and its last `recent` tokens) keeps the `need` largest weights, ties
// to the lower place.  A CTA per (sequence, head) finds the need-th largest by its bits, 11, 11 and 10 at a time: a count of
// the values of each digit, then the digit in which the need-th falls.  Two more passes count and write the places in
// order: a warp owns a run of the middle, so only its totals are exchanged.
struct KeepArgs {
    PagedView c;
    const float* w;     // [n_pages, H_kv, page_size]
    int32_t* keep;      // [batch, H_kv, budget]
    int32_t* new_lens;  // [batch] or null
    int budget, sinks, recent;
};

constexpr int kKeepThreads = 1024, kKeepBins = 2048;

// VEC: weights that a lane reads at a time, 4 where pages are whole runs of 16 bytes.
template <int VEC>
__global__ void __launch_bounds__(kKeepThreads)
paged_keep_kernel(const KeepArgs a, int* status) {
    __shared__ uint32_t hist[kKeepBins], scan[33], found[3];
    const int s = blockIdx.x / a.c.H_kv, head = blockIdx.x - s * a.c.H_kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t cap = (int64_t)a.c.max_pages * a.c.page_size;
    const int len = a.c.kv_lens[s];
    if ((len < 0 || len > cap) && threadIdx.x == 0 && head == 0) report_async(status, kAsyncBadIndex, 0x901);
    const int L = (int)min((int64_t)max(len, 0), cap);
    const int n = min(L, a.budget), recent = min(a.recent, n), sinks = min(a.sinks, n - recent);
    const int lo = sinks, hi = L - recent, need = n - recent - sinks;  // the middle [lo, hi) keeps `need`
    int32_t* out = a.keep + (int64_t)blockIdx.x * a.budget;
    if (a.new_lens != nullptr && threadIdx.x == 0 && head == 0) a.new_lens[s] = n;
    for (int i = threadIdx.x; i < a.budget; i += kKeepThreads) {
        if (i < sinks || (L == n && i < n)) out[i] = i;
        else if (i >= n) out[i] = -1;
        else if (i >= n - recent) out[i] = L - n + i;
    }
    if (L == n || need == 0) return;

    const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
    const uint32_t size = a.c.page_size;
    // a warp's run of places, in steps of 32 VEC from a multiple of VEC
    const int from = lo / VEC * VEC, steps = (hi - from + 32 * VEC - 1) / (32 * VEC), per = (steps + 31) / 32;
    const int run_lo = from + min(steps, warp * per) * 32 * VEC, run_hi = from + min(steps, (warp + 1) * per) * 32 * VEC;
    // keys of places at .. at + VEC - 1; those outside the middle: `in` says
    auto keys_at = [&](int at, uint32_t (&key)[VEC], bool (&in)[VEC]) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) { v[e] = __int_as_float(0x7fc00000); in[e] = at + e >= lo && at + e < hi; }
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

    // ---- the need-th largest key
    uint32_t want = need, prefix = 0;
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
        for (int i = threadIdx.x; i < kKeepBins; i += kKeepThreads) hist[i] = 0;
        __syncthreads();
        for (int at = run_lo + lane * VEC; at < run_hi; at += 32 * VEC) {
            uint32_t key[VEC];
            bool in[VEC];
            keys_at(at, key, in);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (in[e] && (round == 0 || key[e] >> (shift + bits) == prefix)) atomicAdd(&hist[(key[e] >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // digits from the top: two a thread
        const int d = kKeepBins - 1 - 2 * (int)threadIdx.x;
        const uint32_t c0 = hist[d], c1 = hist[d - 1];
        uint32_t all;
        const uint32_t above = block_scan(c0 + c1, scan, &all);
        if (above < want && above + c0 + c1 >= want) {  // (one thread)
            const bool first = above + c0 >= want;
            found[0] = first ? d : d - 1;
            found[1] = want - above - (first ? 0u : c0);
        }
        __syncthreads();
        prefix = round == 0 ? found[0] : (prefix << bits) | found[0];
        want = found[1];
    }
    // ---- kept: keys above `prefix`, and the first `want` of those equal to it
    uint32_t mine_above = 0, mine_equal = 0;
    for (int at = run_lo + lane * VEC; at < run_hi; at += 32 * VEC) {
        uint32_t key[VEC];
        bool in[VEC];
        keys_at(at, key, in);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            mine_above += in[e] && key[e] > prefix;
            mine_equal += in[e] && key[e] == prefix;
        }
    }
    mine_above = __reduce_add_sync(0xffffffffu, mine_above);
    mine_equal = __reduce_add_sync(0xffffffffu, mine_equal);
    uint32_t all;
    uint32_t equal = block_scan(lane == 0 ? mine_equal : 0u, scan, &all);  // equal ones in earlier warps
    equal = __shfl_sync(0xffffffffu, equal, 0);
    const uint32_t take = equal >= want ? 0u : min(mine_equal, want - equal);
    uint32_t rank = block_scan(lane == 0 ? mine_above + take : 0u, scan, &all);
    rank = __shfl_sync(0xffffffffu, rank, 0);
    for (int at0 = run_lo; at0 < run_hi; at0 += 32 * VEC) {
        const int at = at0 + lane * VEC;
        uint32_t key[VEC];
        bool in[VEC];
        keys_at(at, key, in);
        uint32_t eq = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) eq += in[e] && key[e] == prefix;
        uint32_t eq_upto = eq;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t below = __shfl_up_sync(0xffffffffu, eq_upto, o);
            if (lane >= o) eq_upto += below;
        }
        uint32_t order = equal + eq_upto - eq, kept = 0;
        bool stay[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool same = in[e] && key[e] == prefix;
            stay[e] = in[e] && (key[e] > prefix || (same && order < want));
            order += same;
            kept += stay[e];
        }
        uint32_t upto = kept;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t below = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += below;
        }
        uint32_t to = rank + upto - kept;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (stay[e]) out[sinks + to++] = at + e;
        equal += __shfl_sync(0xffffffffu, eq_upto, 31);
        rank += __shfl_sync(0xffffffffu, upto, 31);
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

constexpr int kCompactThreads = 256, kCompactLoads = 8;

// Rows of a pool that places stand at, -1: nowhere.
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
template <class V>
__global__ void __launch_bounds__(kCompactThreads)
paged_compact_kernel(const CompactArgs a, int slices, int* status) {
    const int s = blockIdx.x / a.c.H_kv, head = blockIdx.x - s * a.c.H_kv;
    const int32_t* keep = a.keep + (int64_t)blockIdx.x * a.width;
    const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
    const int64_t len = min((int64_t)max(a.c.kv_lens[s], 0), (int64_t)a.c.max_pages * a.c.page_size);
    const int part = blockIdx.y;
    if (part == 2 * slices) {
        constexpr int RUN = kCompactThreads * kCompactLoads;
        for (int first = 0; first < a.width; first += RUN) {
            float v[kCompactLoads];
            int64_t to[kCompactLoads];
#pragma unroll
            for (int j = 0; j < kCompactLoads; ++j) {
                const int i = first + j * kCompactThreads + (int)threadIdx.x, place = i < a.width ? keep[i] : -1;
                const int64_t row = compact_row(a.c, table, place, len, status);
                const int64_t dst = row >= 0 && place > i ? compact_row(a.c, table, i, len, status) : -1;
                if (place >= 0 && place < i) report_async(status, kAsyncBadIndex, 0xA03);  // (not ascending from 0)
                to[j] = -1;
                if (dst >= 0) {
                    const int64_t off = row % a.c.page_size, off2 = dst % a.c.page_size;
                    v[j] = a.w[(row - off) * a.c.H_kv + (int64_t)head * a.c.page_size + off];
                    to[j] = (dst - off2) * a.c.H_kv + (int64_t)head * a.c.page_size + off2;
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
    const int slice = part >= slices ? part - slices : part;
    const int lanes = a.slice_bytes / (int)sizeof(V), rows = kCompactThreads / lanes;  // rows of a load of the CTA
    const int in_row = threadIdx.x % lanes, row0 = threadIdx.x / lanes;
    const int64_t column = (int64_t)head * a.row_bytes + slice * a.slice_bytes + in_row * (int)sizeof(V);
    const int64_t pitch = (int64_t)a.c.H_kv * a.row_bytes;
    if (pool == nullptr) return;
    for (int first = 0; first < a.width; first += rows * kCompactLoads) {
        V v[kCompactLoads];
        int64_t to[kCompactLoads];
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j) {
            const int i = first + j * rows + row0, place = row0 < rows && i < a.width ? keep[i] : -1;
            const int64_t row = compact_row(a.c, table, place, len, status);
            to[j] = row >= 0 && place > i ? compact_row(a.c, table, i, len, status) : -1;
            if (place >= 0 && place < i) report_async(status, kAsyncBadIndex, 0xA03);  // (not ascending from 0)
            if (to[j] >= 0) v[j] = *reinterpret_cast<const V*>(pool + row * pitch + column);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kCompactLoads; ++j)
            if (to[j] >= 0) *reinterpret_cast<V*>(pool + to[j] * pitch + column) = v[j];
        __syncthreads();
    }
}

}  // namespace msa
