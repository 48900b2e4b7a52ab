// The next token from its logits and a given random number (include/msa.h: msa_sample).
//
// What is kept of a row, in turn: the top_k largest logits; of their probabilities the shortest prefix, largest first, that
// has top_p of their mass; of these the ones of at least min_p times the largest.  The token is the first, in the order of the
// vocabulary, at which the kept probabilities' running sum exceeds u times their sum.  Ties go to the lower index throughout.
//
// Probabilities only matter up to a factor: w = exp((x - max) / T), the largest is 1.  They are held as whole numbers of 2^-42
// (64 bits), so sums are exact in any order - equal calls choose equal tokens - and a border between two tokens moves by less than
// 2^-42 for each token in front of it.  (In 32 bits a border among 10^5 tokens would be off by more than the tokens themselves.)
#pragma once

#include "order.cuh"

namespace msa {

struct SampleArgs {
    const void* logits;
    int64_t stride;
    int vocab;
    const float* u;
    // settings of every row, or of all
    const float* temperatures; const int32_t* top_ks; const float* top_ps; const float* min_ps;
    float temperature; int32_t top_k; float top_p; float min_p;
    int64_t* token;
    float* logprob;
};

constexpr int kSampleThreads = 1024, kSampleBins = 2048, kSampleTable = 256;
constexpr double kSampleOne = 4398046511104.0;  // 2^42

template <class T> __device__ __forceinline__ float logit_at(const T* x, int64_t i);
template <> __device__ __forceinline__ float logit_at(const float* x, int64_t i) { return __ldg(x + i); }
template <> __device__ __forceinline__ float logit_at(const __half* x, int64_t i) { return __half2float(__ldg(x + i)); }
template <> __device__ __forceinline__ float logit_at(const __nv_bfloat16* x, int64_t i) { return __bfloat162float(__ldg(x + i)); }

// 2^42 exp(-d c ln 2) for d >= 0 and c = log2(e) / T, rounded to a whole number: 2^-z = 2^-n 2^(-j/256) 2^-r with z = n + j/256 + r,
// r < 2^-8; 2^(-j/256) from a table, 2^-r by its Taylor series to the fourth power (off by less than 2^-50).  d = infinity: 0.
__device__ __forceinline__ uint64_t sample_weight(double d, double c, const double* table) {
    if (d == 0.0) return (uint64_t)1 << 42;
    const double z = d * c;
    if (!(z < 44.0)) return 0;
    const int k = (int)(z * kSampleTable);
    const double r = (z - (double)k * (1.0 / kSampleTable)) * -0.69314718055994530942;
    const double p = fma(r, fma(r, fma(r, fma(r, 1.0 / 24, 1.0 / 6), 0.5), 1.0), 1.0);
    const double w = table[k & (kSampleTable - 1)] * p;
    return (uint64_t)__double2ull_rn(__hiloint2double(__double2hiint(w) + ((42 - (k >> 8)) << 20), __double2loint(w)));
}

__device__ __forceinline__ uint64_t warp_add64(uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A CTA per row.
template <class T>
__global__ void __launch_bounds__(kSampleThreads)
sample_kernel(const SampleArgs a) {
    __shared__ uint32_t count[kSampleBins], mass_lo[kSampleBins], mass_hi[kSampleBins];
    __shared__ double table[kSampleTable];
    __shared__ uint64_t sums[33];
    __shared__ uint32_t scan[33];
    __shared__ float tops[32];
    __shared__ uint64_t f64[2];
    __shared__ uint32_t f32[3];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int V = a.vocab;
    const float temperature = a.temperatures ? a.temperatures[row] : a.temperature;
    const int top_k = a.top_ks ? a.top_ks[row] : a.top_k;
    const float top_p = a.top_ps ? a.top_ps[row] : a.top_p, min_p = a.min_ps ? a.min_ps[row] : a.min_p;
    const double u = (double)a.u[row];
    // a warp's run of the vocabulary
    const int per = (V + 32 * 32 - 1) / (32 * 32) * 32, run_lo = min(V, warp * per), run_hi = min(V, run_lo + per);

    for (int i = threadIdx.x; i < kSampleTable; i += kSampleThreads) table[i] = exp2((double)-i / kSampleTable);
    float top = -INFINITY;
    bool nan = !(temperature == temperature) || !(u == u);
    for (int i = run_lo + lane; i < run_hi; i += 32) {
        const float v = logit_at(x, i);
        nan |= v != v;
        top = fmaxf(top, v);
    }
    top = warp_max(top);
    if (lane == 0) tops[warp] = top;
    nan = __syncthreads_or(nan) != 0;
    top = warp_max(tops[lane]);
    if (nan || top == -INFINITY) {  // nothing to choose from
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = __int_as_float(0x7fc00000);
        }
        return;
    }
    const bool greedy = !(temperature > 0.f);
    const double c = greedy ? INFINITY : 1.4426950408889634074 / (double)temperature;
    auto below = [&](float v) { return v == top ? 0.0 : (double)top - (double)v; };  // (in 32 bits the difference is rounded)
    auto weight = [&](float v) { return sample_weight(below(v), c, table); };

    // what is kept: keys above `key`, and those equal to it up to index `last`
    uint32_t key = 0;
    int last = V;
    auto kept = [&](float v, int i) {
        const uint32_t k = order_key(v);
        return k > key || (k == key && i <= last);
    };
    // The key at which a running count (or mass), largest first, reaches the target; then the index at which it does.
    auto narrow = [&](bool by_mass, uint64_t target) {
        uint32_t prefix = 0;
        uint64_t want = target;
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
            for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) count[i] = mass_lo[i] = mass_hi[i] = 0;
            __syncthreads();
            for (int i = run_lo + lane; i < run_hi; i += 32) {
                const float v = logit_at(x, i);
                const uint32_t k = order_key(v);
                if (!kept(v, i) || (round > 0 && k >> (shift + bits) != prefix)) continue;
                const uint32_t bin = (k >> shift) & ((1u << bits) - 1);
                atomicAdd(&count[bin], 1u);
                if (by_mass) {
                    const uint64_t w = weight(v);
                    const uint32_t old = atomicAdd(&mass_lo[bin], (uint32_t)w);
                    const uint32_t carry = old + (uint32_t)w < old ? 1u : 0u, high = (uint32_t)(w >> 32) + carry;
                    if (high != 0) atomicAdd(&mass_hi[bin], high);
                }
            }
            __syncthreads();
            // digits from the top, two a thread
            const int d = kSampleBins - 1 - 2 * (int)threadIdx.x;
            const uint64_t c0 = by_mass ? ((uint64_t)mass_hi[d] << 32) + mass_lo[d] : count[d];
            const uint64_t c1 = by_mass ? ((uint64_t)mass_hi[d - 1] << 32) + mass_lo[d - 1] : count[d - 1];
            uint64_t upto = c0 + c1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t before = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += before;
            }
            if (lane == 31) sums[warp] = upto;
            __syncthreads();
            for (int w = 0; w < warp; ++w) upto += sums[w];
            const uint64_t above = upto - c0 - c1;
            if (above < want && upto >= want) {  // (one thread)
                const bool first = above + c0 >= want;
                f32[0] = first ? d : d - 1;
                f64[0] = want - above - (first ? 0 : c0);
            }
            __syncthreads();
            prefix = round == 0 ? f32[0] : (prefix << bits) | f32[0];
            want = f64[0];
        }
        // of the logits equal to the key, as many as are wanted
        uint32_t ties = 0;
        for (int i = run_lo + lane; i < run_hi; i += 32) {
            const float v = logit_at(x, i);
            if (order_key(v) == prefix && kept(v, i)) ++ties;
            if (order_key(v) == prefix) f64[1] = by_mass ? weight(v) : 1;  // (all the same value)
        }
        const uint32_t mine = __reduce_add_sync(0xffffffffu, ties);
        uint32_t all, before = block_scan(lane == 0 ? mine : 0u, scan, &all);
        before = __shfl_sync(0xffffffffu, before, 0);
        const uint64_t one = f64[1];
        const uint64_t needed = one == 0 ? all : (want + one - 1) / one;
        const uint32_t m = (uint32_t)min(needed, (uint64_t)all);  // the m-th tie is the last
        if (m > before && m <= before + mine) {
            uint32_t at = before;
            for (int i0 = run_lo; i0 < run_hi; i0 += 32) {
                const int i = i0 + lane;
                const float v = i < run_hi ? logit_at(x, i) : -INFINITY;
                const bool tie = i < run_hi && order_key(v) == prefix && kept(v, i);
                const unsigned all_ties = __ballot_sync(0xffffffffu, tie);
                if (tie && at + __popc(all_ties & ((1u << lane) - 1)) + 1 == m) f32[1] = i;
                at += __popc(all_ties);
            }
        }
        __syncthreads();
        key = prefix;
        last = (int)f32[1];
    };
    // The sum of what is kept, in each warp's run and in all.
    uint64_t total = 0, before = 0;
    double least = INFINITY;  // largest distance to the top, in units of T, that min_p allows
    auto in = [&](float v, int i) { return kept(v, i) && (v == top || below(v) <= least); };
    auto add_up = [&]() {
        uint64_t mine = 0;
        for (int i = run_lo + lane; i < run_hi; i += 32) {
            const float v = logit_at(x, i);
            if (in(v, i)) mine += weight(v);
        }
        mine = warp_add64(mine);
        __syncthreads();
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
        total = before = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) before += sums[w];
            total += sums[w];
        }
        return mine;
    };
    if (greedy) narrow(false, 1);
    else {
        if (top_k > 0 && top_k < V) narrow(false, top_k);
        if (top_p < 1.f) {
            add_up();
            const double target = (double)total * (double)fmaxf(top_p, 0.f);
            // whole numbers: reaching the target is reaching the next whole number
            narrow(true, max((uint64_t)1, (uint64_t)ceil(target)));
        }
        if (min_p > 0.f) least = -log((double)min_p) * (double)temperature;
    }
    const uint64_t mine = add_up();
    const double target = u * (double)total;
    // The first index whose running sum exceeds the target (the last kept one, where u is 1 or more).
    if (threadIdx.x == 0) f32[2] = 0;
    __syncthreads();
    const bool here = mine > 0 && (double)before <= target && (double)(before + mine) > target;
    const bool beyond = mine > 0 && before + mine == total && target >= (double)total;
    if (here || beyond || (mine > 0 && before == 0 && target < 0)) {
        uint64_t sum = before;
        int choice = -1;
        float value = 0.f;
        for (int i0 = run_lo; i0 < run_hi && choice < 0; i0 += 32) {
            const int i = i0 + lane;
            const float v = i < run_hi ? logit_at(x, i) : -INFINITY;
            const uint64_t w = i < run_hi && in(v, i) ? weight(v) : 0;
            uint64_t upto = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t b = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += b;
            }
            upto += sum;
            const unsigned hit = __ballot_sync(0xffffffffu, w > 0 && ((double)upto > target || upto == total));
            if (hit != 0) {
                choice = i0 + __ffs(hit) - 1;
                value = __shfl_sync(0xffffffffu, v, __ffs(hit) - 1);
            }
            sum = __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) {
            a.token[row] = choice;
            if (a.logprob)
                a.logprob[row] = greedy ? 0.f : (float)((value == top ? 0.0 : -below(value) / (double)temperature) - log((double)total / kSampleOne));
        }
    }
}

}  // namespace msa
