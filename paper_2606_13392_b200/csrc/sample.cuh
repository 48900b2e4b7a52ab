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

#include <cooperative_groups.h>

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

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32, kSampleTable = 1024;
constexpr int kSampleBins = 512;                // of equal width in log w
constexpr int kSampleDigits = 2048;             // sample_slow: values of eleven bits
constexpr int kSampleCtas = 8;                  // of a row, at most
constexpr int kSampleList = 4096, kSampleSort = 2048, kSamplePairs = 128;  // places of the list; tokens that are sorted, compared in pairs
constexpr int kSampleBits = 42;
constexpr double kSampleOne = 4398046511104.0;  // 2^42
constexpr float kSampleReach = 43.f;            // 2^-43 of the largest is no whole number any more

// Larger of two, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Two or four bytes of a row: 16 bytes at a time.
template <class T> struct Logits;
template <> struct Logits<float> {
    static constexpr int E = 4;
    static constexpr bool HALF = false;
    static __device__ __forceinline__ void widen(const uint4& r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ float largest(const uint4& r) {
        return max_nan(max_nan(__uint_as_float(r.x), __uint_as_float(r.y)), max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
    }
};
template <> struct Logits<__half> {
    static constexpr int E = 8;
    static constexpr bool HALF = true;
    static __device__ __forceinline__ void widen(const uint4& r, float (&v)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float largest(const uint4& r) {
        const __half2* h = reinterpret_cast<const __half2*>(&r);
        const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return max_nan(__low2float(m), __high2float(m));
    }
};
template <> struct Logits<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr bool HALF = false;
    static __device__ __forceinline__ void widen(const uint4& r, float (&v)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = bf16x2_to_float2(w[i]);
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float largest(const uint4& r) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
        const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return max_nan(__low2float(m), __high2float(m));
    }
};

// A row as whole 16-byte pieces of memory: its first value is number `skip` of the first piece.  Values of a piece that are not
// the row's read as -infinity (and are not loaded).
template <class T>
struct SampleRow {
    static constexpr int E = Logits<T>::E;
    const T* x;
    int vocab, skip, pieces;
    __device__ SampleRow(const T* row, int v) : x(row), vocab(v) {
        skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        pieces = (skip + v + E - 1) / E;
    }
    __device__ __forceinline__ int index(int piece) const { return piece * E - skip; }  // of the piece's first value
    __device__ __forceinline__ uint4 load(int piece) const {
        const int at = index(piece);
        if (at >= 0 && at + E <= vocab) return __ldg(reinterpret_cast<const uint4*>(x + at));
        alignas(16) T v[E];  // (read as one below)
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at + e >= 0 && at + e < vocab ? __ldg(x + at + e) : T(-INFINITY);
        return *reinterpret_cast<const uint4*>(v);
    }
    static __device__ __forceinline__ uint4 nothing() {
        const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : (E == 8 && Logits<T>::HALF ? 0xFC00FC00u : 0xFF80FF80u);
        return make_uint4(w, w, w, w);
    }
};

// Pieces [lo, hi) of a warp: a run of the row, lanes side by side, U in flight (few where f is long: a loop that does not fit the
// instruction cache is what slows these passes most); U = 0: one, while the next two are on their way.  f(piece, index of its first value) is called by
// all lanes of the warp (beyond the run: with -infinities).
template <int U, class T, class F>
__device__ __forceinline__ void sample_pieces(const SampleRow<T>& row, int lo, int hi, F f) {
    const int lane = threadIdx.x & 31;
    auto load = [&](int p) { return p < hi ? row.load(p) : SampleRow<T>::nothing(); };
    if constexpr (U == 0) {
        uint4 next[2] = {load(lo + lane), load(lo + 32 + lane)};
        for (int p0 = lo; p0 < hi; p0 += 32) {
            const uint4 raw = next[0];
            next[0] = next[1];
            next[1] = load(p0 + 64 + lane);
            f(raw, row.index(p0 + lane));
        }
    } else {
        for (int p0 = lo; p0 < hi; p0 += 32 * U) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = load(p0 + u * 32 + lane);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p0 + u * 32 < hi) f(raw[u], row.index(p0 + u * 32 + lane));
        }
    }
}
// The same with the values as floats.
template <int U = 1, class T, class F>
__device__ __forceinline__ void sample_run(const SampleRow<T>& row, int lo, int hi, F f) {
    sample_pieces<U>(row, lo, hi, [&](const uint4& raw, int at) {
        float v[SampleRow<T>::E];
        Logits<T>::widen(raw, v);
        f(v, at);
    });
}

// What a token's weight and place in the order are computed from.
struct SampleScale {
    float top, c32;         // largest logit; c in 32 bits, for bins
    double c, tc, ct, tct;  // log2(e) / T; top c; c and top c times the table's size, the latter with 1.5 2^52 in front
    const double* table;
    static constexpr double kFront = 6755399441055744.0;  // 1.5 2^52: a sum with it has the nearest whole number in its last bits

    __device__ __forceinline__ SampleScale(float top_, double T, const double* table_) : top(top_), table(table_) {
        c = 1.4426950408889634074 / T;
        c32 = fminf((float)c, 3e38f);
        tc = (double)top * c;
        ct = c * kSampleTable;
        tct = fma((double)top, ct, kFront);  // (rounded once, or the top itself could come out half a step before itself)
    }
    // Distance to the top (in 32 bits it would be rounded); a top of infinity comes with sample_slow only.
    __device__ __forceinline__ double below(float v) const { return (double)top - (double)v; }
    // 2^42 2^(-k/1024) 2^-r to the nearest whole number, `some` is false: 0.  2^(-k/1024) from a table and an exponent, 2^-r, |r| <=
    // 2^-10, by its Taylor series to the third power (off by less than 2^-46); the rounding by adding 2^52.
    __device__ __forceinline__ uint64_t power(int k, double r, bool some) const {
        constexpr double L = -0.69314718055994530942;
        const double p = fma(r, fma(r, fma(r, L * L * L / 6, L * L / 2), L), 1.0);
        const double root = table[k & (kSampleTable - 1)];
        const double scaled = __hiloint2double(__double2hiint(root) + ((kSampleBits - (k >> 10)) << 20), __double2loint(root));
        const uint64_t whole = (uint64_t)__double_as_longlong(fma(scaled, p, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
        return some ? whole : 0;  // (no branch: what is computed beyond the reach is not used)
    }
    // Weight at a distance d >= 0 of the top: z = d c = k / 1024 + r.  From z = 43 on (infinity, too; NaN): 0.
    __device__ __forceinline__ uint64_t weight(double d) const {
        const double z = d * c, t = fma(z, (double)kSampleTable, kFront);
        return power(__double2loint(t), fma(t - kFront, -1.0 / kSampleTable, z), z < (double)kSampleReach);
    }
    // The same of a logit, for |top c| < 2^20: z = top c - v c with one rounding.  (That of top c is the same for all, and so a common
    // factor of all weights, of less than 1 + 2^-33.)
    __device__ __forceinline__ uint64_t weight_of(float v) const {
        const double x = (double)v, t = fma(x, -ct, tct);
        const int k = __double2loint(t);  // whole and small where the upper half is that of 1.5 2^52
        const bool some = __double2hiint(t) == 0x43380000 && (uint32_t)k < (uint32_t)(kSampleReach * kSampleTable);
        return power(k, fma(x, -c, fma(t - kFront, -1.0 / kSampleTable, tc)), some);
    }
    // Distance to the top in 32 bits, in units of the bins' axis (log2 of the weight).  Its operations, and those that make bins of it,
    // are named: contracted in one pass over the row and not in another, a logit would change its bin.
    __device__ __forceinline__ float distance(float v) const { return __fmul_rn(__fsub_rn(top, v), c32); }
    // Bin of a logit, larger logits in lower bins; kSampleBins: its weight is 0.
    __device__ __forceinline__ int bin(float v) const {
        const float z = distance(v);
        return z < kSampleReach ? min((int)__fmul_rn(z, kSampleBins / kSampleReach), kSampleBins - 1) : kSampleBins;
    }
};

__device__ __forceinline__ uint64_t warp_add64(uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint64_t warp_upto64(uint64_t v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t b = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v += b;
    }
    return v;
}
// Inclusive sum over the CTA's threads; the total in s[kSampleWarps].  s: kSampleWarps + 1 words of shared memory.
__device__ __forceinline__ uint64_t block_upto64(uint64_t v, uint64_t* s) {
    const int warp = threadIdx.x >> 5;
    v = warp_upto64(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) s[warp] = v;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSampleWarps; ++w) {
        if (w < warp) before += s[w];
        all += s[w];
    }
    if (threadIdx.x == 0) s[kSampleWarps] = all;
    __syncthreads();
    return v + before;
}

struct SampleSmem {
    double table[kSampleTable], root[64];
    uint32_t count[kSampleBins], mass_lo[kSampleBins], mass_hi[kSampleBins];
    union {
        uint32_t counts[kSampleCtas][kSampleBins];  // of every CTA
        uint64_t work[kSampleSort];                 // the list, packed
    };
    union {
        uint64_t masses[kSampleCtas][kSampleBins];  // of every CTA
        uint64_t list[kSampleList];                 // (key, ~index): larger first means larger logit, then lower index; a part for each CTA
        struct { uint32_t count[kSampleDigits], lo[kSampleDigits], hi[kSampleDigits]; } digits;  // sample_slow
    };
    uint64_t pair_w[kSamplePairs];
    uint64_t sums[kSampleWarps + 1];
    uint32_t scan[33];
    float tops[kSampleWarps];
    uint32_t listed;
    // what the CTAs tell one another (each is written once a row)
    struct { float top; int nan; } said;
    uint64_t totals[kSampleCtas], aboves[kSampleCtas], parts[kSampleCtas];
    uint32_t sizes[kSampleCtas];
    uint32_t last_key;
    int last_index;
    // results of a search by one thread
    uint64_t found64[2];
    uint32_t found32[3];
};

// Sorts list[0, n) in descending order (up to the next power of two, filled with zeros).  Short lists a value a thread, whose
// partners in the same warp trade places in registers.
__device__ inline void sample_sort(uint64_t* list, int n) {
    int size = 32;
    while (size < n) size *= 2;
    if (size <= kSampleThreads) {
        const int i = threadIdx.x;
        uint64_t x = i < n ? list[i] : 0;
        __syncthreads();
        for (int k = 2; k <= size; k *= 2) {
            int j = k / 2;
            for (; j >= 32; j /= 2) {
                if (i < size) list[i] = x;
                __syncthreads();
                const uint64_t y = i < size ? list[i ^ j] : 0;
                __syncthreads();
                x = (x > y) == (((i & k) == 0) == ((i & j) == 0)) ? x : y;
            }
            if (i < size)
                for (; j > 0; j /= 2) {
                    const uint64_t y = __shfl_xor_sync(0xffffffffu, x, j);
                    x = (x > y) == (((i & k) == 0) == ((i & j) == 0)) ? x : y;  // (the larger of the two, or the smaller)
                }
        }
        if (i < size) list[i] = x;
        __syncthreads();
        return;
    }
    for (int i = n + threadIdx.x; i < size; i += kSampleThreads) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            for (int t = threadIdx.x; t < size / 2; t += kSampleThreads) {
                const int a = 2 * t - (t & (j - 1)), b = a + j;
                const uint64_t x = list[a], y = list[b];
                if ((x < y) == ((a & k) == 0)) { list[a] = y; list[b] = x; }
            }
            __syncthreads();
        }
    }
}

__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key); }

// ---------------------------------------------------------------- any row, by one CTA
// Whatever is kept, however many are equal: thresholds by the bits of the logits, 11, 11 and 10 at a time, each a pass over
// the row that adds up counts or weights of the digits; then the index among equal ones.  For rows that the lists below do not hold.
template <class T>
__device__ __noinline__ void sample_slow(const SampleArgs a, int64_t row_number, const SampleRow<T> row, const SampleScale sc, double least, SampleSmem& sm,
                                   bool greedy, int top_k, float top_p, double temperature, double u) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = (row.pieces + 32 * kSampleWarps - 1) / (32 * kSampleWarps) * 32;
    const int run_lo = min(row.pieces, warp * per), run_hi = min(row.pieces, run_lo + per);
    constexpr int E = SampleRow<T>::E;
    // what is kept: keys above `key`, and those equal to it up to index `last`
    uint32_t key = 0;
    int last = row.vocab;
    auto kept = [&](float v, int i) {
        const uint32_t k = order_key(v);
        return v > -INFINITY && (k > key || (k == key && i <= last));
    };
    auto below = [&](float v) { return v == sc.top ? 0.0 : sc.below(v); };  // (the top may be infinite)
    auto weight_of = [&](float v) { return sc.weight(below(v)); };
    // (the target is at most all that there is: a row may have fewer logits to choose from than top_k)
    auto narrow = [&](bool by_mass, uint64_t target) {
        uint32_t prefix = 0;
        uint64_t want = target;
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
            __syncthreads();
            for (int i = threadIdx.x; i < kSampleDigits; i += kSampleThreads) sm.digits.count[i] = sm.digits.lo[i] = sm.digits.hi[i] = 0;
            __syncthreads();
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t k = order_key(v[e]);
                    if (!kept(v[e], at + e) || (round > 0 && k >> (shift + bits) != prefix)) continue;
                    const uint32_t bin = (k >> shift) & ((1u << bits) - 1);
                    atomicAdd(&sm.digits.count[bin], 1u);
                    if (by_mass) {
                        const uint64_t w = weight_of(v[e]);
                        const uint32_t old = atomicAdd(&sm.digits.lo[bin], (uint32_t)w);
                        const uint32_t high = (uint32_t)(w >> 32) + (old + (uint32_t)w < old ? 1u : 0u);
                        if (high != 0) atomicAdd(&sm.digits.hi[bin], high);
                    }
                }
            });
            __syncthreads();
            uint64_t c[4], mine = 0;  // digits from the top, four a thread
            const int d = kSampleDigits - 1 - 4 * (int)threadIdx.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = by_mass ? ((uint64_t)sm.digits.hi[d - j] << 32) + sm.digits.lo[d - j] : sm.digits.count[d - j];
                mine += c[j];
            }
            uint64_t above = block_upto64(mine, sm.sums) - mine;
            if (round == 0) want = min(want, sm.sums[kSampleWarps]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (above < want && above + c[j] >= want) { sm.found32[0] = d - j; sm.found64[0] = want - above; }  // (one thread)
                above += c[j];
            }
            __syncthreads();
            prefix = round == 0 ? sm.found32[0] : (prefix << bits) | sm.found32[0];
            want = sm.found64[0];
        }
        // of the logits equal to the key, as many as are wanted
        uint32_t ties = 0;
        sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
#pragma unroll
            for (int e = 0; e < E; ++e) ties += order_key(v[e]) == prefix && kept(v[e], at + e);
        });
        const uint64_t one = by_mass ? weight_of(key_value(prefix)) : 1;
        const uint32_t mine = __reduce_add_sync(0xffffffffu, ties);
        uint32_t all, before = block_scan(lane == 0 ? mine : 0u, sm.scan, &all);
        before = __shfl_sync(0xffffffffu, before, 0);
        const uint64_t needed = one == 0 ? all : (want + one - 1) / one;
        const uint32_t m = (uint32_t)min(needed, (uint64_t)all);  // the m-th tie is the last
        if (m > before && m <= before + mine) {
            uint32_t at_tie = before;
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
                uint32_t here = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) here += order_key(v[e]) == prefix && kept(v[e], at + e);
                uint32_t upto = here;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t b = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += b;
                }
                uint32_t n = at_tie + upto - here;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (order_key(v[e]) == prefix && kept(v[e], at + e) && ++n == m) sm.found32[1] = at + e;
                at_tie += __shfl_sync(0xffffffffu, upto, 31);
            });
        }
        __syncthreads();
        key = prefix;
        last = (int)sm.found32[1];
    };
    auto in = [&](float v, int i) { return kept(v, i) && below(v) <= least; };
    auto add_up = [&]() {
        uint64_t mine = 0;
        sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (in(v[e], at + e)) mine += weight_of(v[e]);
        });
        return warp_add64(mine);
    };
    if (greedy) narrow(false, 1);
    else {
        if (top_k > 0 && top_k < row.vocab) narrow(false, top_k);
        if (top_p < 1.f) {
            uint64_t mine = 0;
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (kept(v[e], at + e)) mine += weight_of(v[e]);
            });
            block_upto64(mine, sm.sums);
            const double target = (double)sm.sums[kSampleWarps] * (double)fmaxf(top_p, 0.f);
            narrow(true, max((uint64_t)1, (uint64_t)ceil(target)));  // whole numbers: reaching the target is reaching the next one
        }
    }
    const uint64_t mine = add_up();
    const uint64_t before = block_upto64(lane == 0 ? mine : 0, sm.sums) - (lane == 0 ? mine : 0);
    const uint64_t start = __shfl_sync(0xffffffffu, before, 0), total = sm.sums[kSampleWarps];
    const double target = u * (double)total;
    uint64_t sum = start;
    if (mine > 0 && ((double)(start + mine) > target || start + mine == total) && ((double)start <= target || start == 0)) {
        bool done = false;
        sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
            if (done) return;
            uint64_t w[E], here = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) { w[e] = in(v[e], at + e) ? weight_of(v[e]) : 0; here += w[e]; }
            const uint64_t upto = warp_upto64(here);
            uint64_t n = sum + upto - here;
            const bool mine_is = here > 0 && ((double)(n + here) > target || n + here == total);
            const unsigned hit = __ballot_sync(0xffffffffu, mine_is);
            if (hit != 0) {
                done = true;
                if (lane == __ffs(hit) - 1) {
                    bool chosen = false;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        n += w[e];
                        if (!chosen && w[e] > 0 && ((double)n > target || n == total)) {
                            chosen = true;
                            a.token[row_number] = at + e;
                            if (a.logprob)
                                a.logprob[row_number] = greedy ? 0.f : (float)(-below(v[e]) / temperature - log((double)total / kSampleOne));
                        }
                    }
                }
            }
            sum += __shfl_sync(0xffffffffu, upto, 31);
        });
    }
}

// ---------------------------------------------------------------- the rows
// A cluster of CTAs per row (one CTA where there are many rows), each with a run of it: a pass for the maximum; then
//   top_k: the threads' own maxima, which that pass has left, are counted in bins of equal width in log w; the bin in which the
//          count reaches k is a bound that the k largest logits reach, and few others.  (All logits are counted, where the threads
//          are not many more than k.)  The tokens that reach it go to a list in the first CTA, which cuts it and chooses from it.
//   top_p alone: the counts of all logits bound the weight of each bin, and so the bins where the nucleus may end; a pass adds up
//          the weights exactly, of the row, and in finer bins between the bounds.  Those of the finer bin in which it ends are
//          listed, to find its last token, and the choice is made as without filters; or all of a nucleus of a few, and it is made there.
//   no filters: every warp adds up its run, and the one that the target falls into finds the token.
// Measured: one row of 131072 with top_k and top_p 11 us (five meetings of the cluster and a short list, 4 - 6 thousand cycles each);
// 512 of 65536 with both 39 us; 96 of 100003 whose settings differ 55 - 58 us (the few without top_k); a flat nucleus of
// 33 rows of 50001 41 us; 256 whole rows of 131072 in fp32 91 us (the row is read twice, and 64-bit arithmetic).
// Where the cycles go, long rows: 30 instructions, 8 of them in 64 bits, a weight, two passes of weights for a nucleus.  Loops that unroll
// more than a piece of 16 bytes leave the instruction cache (512 rows of 65536: 55 us with four).
template <class T>
__global__ void __launch_bounds__(kSampleThreads, 2)
sample_kernel(const SampleArgs a) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint8_t sample_smem[];
    SampleSmem& sm = *reinterpret_cast<SampleSmem*>(sample_smem);
    constexpr int E = SampleRow<T>::E;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / ctas;
    const SampleRow<T> row(static_cast<const T*>(a.logits) + r * a.stride, a.vocab);
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    const int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    const float top_p = a.top_ps ? a.top_ps[r] : a.top_p, min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const double u = fmax((double)a.u[r], 0.0) + 0.0 * a.u[r];  // (a NaN stays one)
    // a warp's run of the row's pieces
    const int warps = ctas * kSampleWarps, per = (row.pieces + 32 * warps - 1) / (32 * warps) * 32;
    const int run_lo = min(row.pieces, (rank * kSampleWarps + warp) * per), run_hi = min(row.pieces, run_lo + per);
    auto sync = [&]() {  // of the row's CTAs
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    };

    // 2^(-i/1024) from 2^(-i/32) and 2^(-i/1024) of the first 32
    if (threadIdx.x < 64) sm.root[threadIdx.x] = exp2((threadIdx.x < 32 ? (double)threadIdx.x / -32 : (double)(threadIdx.x - 32) / -1024));
    for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) sm.count[i] = sm.mass_lo[i] = sm.mass_hi[i] = 0;
    if (threadIdx.x == 0) sm.listed = 0;

    // ---- the largest logit; this thread's own
    float own_top = -INFINITY, top;
    {
        sample_pieces<4>(row, run_lo, run_hi, [&](const uint4& raw, int) { own_top = max_nan(own_top, Logits<T>::largest(raw)); });
        bool nan = __syncthreads_or(own_top != own_top) != 0;
        top = warp_max(own_top);
        if (lane == 0) sm.tops[warp] = top;
        for (int i = threadIdx.x; i < kSampleTable; i += kSampleThreads) sm.table[i] = sm.root[i >> 5] * sm.root[32 + (i & 31)];
        __syncthreads();
        top = warp_max(sm.tops[lane % kSampleWarps]);
        if (ctas > 1) {
            if (threadIdx.x == 0) { sm.said.top = top; sm.said.nan = nan; }
            cluster.sync();
            const auto* other = cluster.map_shared_rank(&sm, lane % ctas);
            top = warp_max(other->said.top);
            nan = __any_sync(0xffffffffu, other->said.nan != 0);
        }
        // (a filter that is not a number filters nothing that could be meant; the largest logit asks for none)
        nan |= !(temperature == temperature) || !(u == u) || (temperature > 0.f && !(top_p == top_p && min_p == min_p));
        if (nan || top == -INFINITY) {  // nothing to choose from
            if (threadIdx.x == 0 && rank == 0) {
                a.token[r] = -1;
                if (a.logprob) a.logprob[r] = __int_as_float(0x7fc00000);
            }
            if (ctas > 1) cluster.sync();  // (the others may still read what this CTA said)
            return;
        }
    }
    const bool greedy = !(temperature > 0.f);
    const double T_ = greedy ? 1.0 : (double)temperature;
    const SampleScale sc(top, T_, sm.table);
    // (at an infinite T a min_p of one asks for zero times infinity: all are as likely as the largest)
    const double least = !greedy && min_p > 0.f && (min_p != 1.f || T_ < INFINITY) ? fmax(0.0, -log((double)min_p) * T_) : INFINITY;
    const int k = greedy ? 1 : top_k;
    bool by_k = k > 0 && k < a.vocab;
    const bool by_p = !greedy && top_p < 1.f;
    const double p = (double)fmaxf(top_p, 0.f);
    const bool tame = fabs(sc.tc) < 1048576.0;  // (weight_of; a top of infinity is not)
    static_assert(kSampleBins == kSampleThreads, "a bin a thread");
    const int b0 = threadIdx.x;

    // The row's count of this thread's bin: every CTA hands its counts to the others.
    auto counted = [&]() {
        __syncthreads();
        if (ctas == 1) return sm.count[b0];
        const uint32_t mine = sm.count[b0];
        for (int c = 0; c < ctas; ++c) *cluster.map_shared_rank(&sm.counts[rank][b0], c) = mine;
        cluster.sync();
        uint32_t n = 0;
        for (int c = 0; c < ctas; ++c) n += sm.counts[c][b0];
        return n;
    };
    // The bin in which a count from the top reaches k: to found32[0], the count up to its end to found32[1].
    auto bin_of_count = [&](uint32_t n, uint32_t* all) {
        const uint32_t upto = block_scan(n, sm.scan, all);
        if (upto < (uint32_t)k && upto + n >= (uint32_t)k) { sm.found32[0] = b0; sm.found32[1] = upto + n; }  // (one thread)
        __syncthreads();
        return upto;
    };

    enum { kAll, kList, kBin, kSlow };
    int mode = kAll;
    // What is listed: top_k: bins up to `end`.  top_p: of the finer bins, `finer` times the distance from `from` on and below
    // `to`, number `end`, or that and all before it.
    float from = 0.f, to = INFINITY, finer = 0.f;
    int end = 0;
    uint64_t whole = 0, above = 0;      // weight of the row, of what comes before the list
    auto finer_bin = [&](float z) { return min((int)__fmul_rn(__fsub_rn(z, from), finer), kSampleBins - 1); };
    constexpr float kWidth = kSampleReach / kSampleBins;
    // Twice as many threads as k, at least, or most of what they would list is not wanted.
    bool by_maxima = by_k && tame && (int64_t)k * 2 <= (int64_t)ctas * kSampleThreads;
    if (by_maxima) {
        const int b = sc.bin(own_top);
        if (b < kSampleBins) atomicAdd(&sm.count[b], 1u);
        uint32_t all;
        bin_of_count(counted(), &all);
        by_maxima = all >= (uint32_t)k;
        if (by_maxima) {
            mode = kList;
            end = (int)sm.found32[0];
        } else {  // the threads' maxima are too few: count all
            sync();
            sm.count[b0] = 0;
            __syncthreads();
        }
    }
    if (!tame) mode = kSlow;
    else if (!by_maxima && (by_k || by_p)) {
        sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int b = sc.bin(v[e]);
                if (b < kSampleBins) atomicAdd(&sm.count[b], 1u);
            }
        });
        const uint32_t n = counted();
        uint32_t all;
        const uint32_t earlier_n = bin_of_count(n, &all);
        by_k = by_k && (uint32_t)k < all;  // (the rest weighs nothing)
        if (by_k) {
            mode = sm.found32[1] <= kSampleSort ? kList : kSlow;
            end = (int)sm.found32[0];
        } else if (by_p) {
            // Bounds of the weight up to each bin, and of what comes behind it: a logit of bin b weighs 2^-(b+1)h to 2^-bh, h the
            // width (and 10^-5 for the 32-bit arithmetic of the bins).  The nucleus ends where what comes behind is at most (1 -
            // top_p) / top_p of what it holds.
            const double w = (double)exp2f(-(float)b0 * kWidth) * n;
            // (in whole numbers, for the scan: 2^-30 of the largest, to the safe side)
            const uint64_t low = (uint64_t)(w * 0.9434 * 0.99997 * 1073741824.0), high = (uint64_t)(w * 1.00003 * 1073741824.0) + 1;  // 2^-h
            static_assert(kSampleBins == 512, "the factor is 2^(-43/512), a little less");
            const uint64_t low_upto = block_upto64(low, sm.sums), low_all = sm.sums[kSampleWarps];
            const uint64_t high_upto = block_upto64(high, sm.sums), high_all = sm.sums[kSampleWarps];
            auto ends = [&](uint64_t behind, uint64_t held) { return p * (double)behind <= (1.0 - p) * (double)held; };
            if (threadIdx.x == 0) { sm.found32[0] = 0; sm.found32[1] = kSampleBins; }
            __syncthreads();
            // the first bin that may hold the end, the first that certainly reaches it
            if (ends(low_all - low_upto, high_upto) && (b0 == 0 || !ends(low_all - (low_upto - low), high_upto - high))) sm.found32[0] = b0;
            if (ends(high_all - high_upto, low_upto) && (b0 == 0 || !ends(high_all - (high_upto - high), low_upto - low))) sm.found32[1] = b0 + 1;
            __syncthreads();
            from = (float)sm.found32[0] * kWidth;
            if (sm.found32[1] < kSampleBins) to = (float)sm.found32[1] * kWidth;
            finer = (float)kSampleBins / ((float)(sm.found32[1] - sm.found32[0]) * kWidth);
            // ---- exact weights: of the row, of what comes before `from`, and in finer bins between `from` and `to`
            uint64_t total = 0, earlier = 0;
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint64_t w = sc.weight_of(v[e]);
                    const float z = sc.distance(v[e]);
                    total += w;
                    if (z < from) earlier += w;
                    else if (z < to && w > 0) {
                        const int b = finer_bin(z);
                        const uint32_t old = atomicAdd(&sm.mass_lo[b], (uint32_t)w);
                        const uint32_t up = (uint32_t)(w >> 32) + (old + (uint32_t)w < old ? 1u : 0u);
                        if (up != 0) atomicAdd(&sm.mass_hi[b], up);
                    }
                }
            });
            block_upto64(total, sm.sums);
            const uint64_t cta_total = sm.sums[kSampleWarps];
            block_upto64(earlier, sm.sums);
            const uint64_t cta_earlier = sm.sums[kSampleWarps];
            uint64_t mass = ((uint64_t)sm.mass_hi[b0] << 32) + sm.mass_lo[b0];
            whole = cta_total;
            above = cta_earlier;
            if (ctas > 1) {
                for (int c = 0; c < ctas; ++c) *cluster.map_shared_rank(&sm.masses[rank][b0], c) = mass;
                if (threadIdx.x < ctas) {
                    auto* other = cluster.map_shared_rank(&sm, threadIdx.x);
                    other->totals[rank] = cta_total;
                    other->aboves[rank] = cta_earlier;
                }
                cluster.sync();
                mass = whole = above = 0;
                for (int c = 0; c < ctas; ++c) { mass += sm.masses[c][b0]; whole += sm.totals[c]; above += sm.aboves[c]; }
            }
            const uint64_t upto = above + block_upto64(mass, sm.sums);
            const uint64_t goal = max((uint64_t)1, (uint64_t)ceil(p * (double)whole));
            if (threadIdx.x == 0) sm.found32[2] = 0xFFFFFFFFu;
            __syncthreads();
            if (upto >= goal && upto - mass < goal) { sm.found32[2] = b0; sm.found64[0] = upto - mass; }  // (one thread)
            __syncthreads();
            end = (int)sm.found32[2];
            mode = end >= 0 ? kBin : kSlow;
            above = sm.found64[0];
            // the tokens up to the bin of the counts in which the finer bin ends: a few? then all are listed
            const float at = from + (float)(end + 1) / finer;
            if (mode == kBin && (float)b0 * kWidth <= at && (float)(b0 + 1) * kWidth > at && earlier_n + n <= kSamplePairs) sm.found32[1] = 0xFFFFFFFFu;
            __syncthreads();
            if (sm.found32[1] == 0xFFFFFFFFu) {
                mode = kList;
                above = 0;
            }
        }
    }
    // Nobody reads another CTA's memory from here on, before the next meeting.
    if (mode == kSlow) {
        sync();
        if (rank == 0) sample_slow<T>(a, r, row, sc, least, sm, greedy, top_k, top_p, T_, u);
        return;
    }

    uint32_t last_key = 0;
    int last_index = a.vocab;
    auto falls_to = [&](uint64_t start, uint64_t n, double target, uint64_t total) {
        // Does the choice fall to weights [start, start + n)?  (The last kept token, where rounding or a u of 1 or more leaves none.)
        return n > 0 && ((double)(start + n) > target || start + n == total) && ((double)start <= target || start == 0);
    };
    auto choose = [&](int index, float v, uint64_t total) {
        a.token[r] = index;
        if (a.logprob) a.logprob[r] = greedy ? 0.f : (float)(-sc.below(v) / T_ - log((double)total / kSampleOne));
    };
    if (mode != kAll) {
        // ---- the list, in the first CTA, a part for each CTA
        if (!by_k && ctas > 1) cluster.sync();  // (it takes the place of the finer bins' weights, which have been read)
        const int part = kSampleList / ctas;
        uint64_t* mine = cluster.map_shared_rank(sm.list, 0) + rank * part;
        auto wanted = [&](float v) {
            if (by_k) return sc.bin(v) <= end;
            const float z = sc.distance(v);
            const int b = z < from ? -1 : (z < to ? finer_bin(z) : kSampleBins);
            return mode == kBin ? b == end : b <= end;
        };
        // (logits at the far end of what is wanted, or a little below: most pieces have none)
        const float z_end = by_k ? (float)(end + 1) * kWidth : from + (float)(end + 1) / finer;
        const float least_listed = sc.top - z_end / sc.c32 * 1.0001f - 1e-6f * fabsf(sc.top);
        sample_pieces<1>(row, run_lo, run_hi, [&](const uint4& raw, int at) {
            if (!(Logits<T>::largest(raw) >= least_listed)) return;
            float v[E];
            Logits<T>::widen(raw, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (v[e] >= least_listed && wanted(v[e])) {
                    const uint32_t n = atomicAdd(&sm.listed, 1u);
                    if (n < (uint32_t)part) mine[n] = (uint64_t)order_key(v[e]) << 32 | (uint32_t)~(at + e);
                }
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) *cluster.map_shared_rank(&sm.sizes[rank], 0) = sm.listed;
        sync();
        if (mode == kList && rank > 0) return;
        if (rank == 0) {
            uint32_t size = 0, first[kSampleCtas + 1];
            bool fits = true;
#pragma unroll
            for (int c = 0; c < kSampleCtas; ++c) {
                const uint32_t n = c < ctas ? sm.sizes[c] : 0;
                fits &= n <= (uint32_t)part;
                first[c] = size;
                size += n;
            }
            fits &= size <= kSampleSort;
            if (threadIdx.x == 0) sm.listed = fits ? 0 : 1;  // (for the others, below)
            if (!fits) {
                if (mode == kBin) { sync(); sync(); }  // (the others learn of it, and have read it)
                __syncthreads();
                sample_slow<T>(a, r, row, sc, least, sm, greedy, top_k, top_p, T_, u);
                return;
            }
            for (uint32_t i = threadIdx.x; i < size; i += kSampleThreads) {
                int c = 0;
#pragma unroll
                for (int j = 1; j < kSampleCtas; ++j) c += j < ctas && i >= first[j];
                uint32_t start = 0;
#pragma unroll
                for (int j = 0; j < kSampleCtas; ++j) start = j == c ? first[j] : start;
                sm.work[i] = sm.list[c * part + (i - start)];
            }
            __syncthreads();
            const uint32_t limit = by_k ? min((uint32_t)k, size) : size;
            uint64_t* list = sm.work;
            if (size <= kSamplePairs) {
                // ---- short: what comes before a token is found by comparing it with all others, four threads a token
                if (threadIdx.x < size) sm.pair_w[threadIdx.x] = sc.weight_of(key_value((uint32_t)(list[threadIdx.x] >> 32)));
                __syncthreads();
                const uint32_t i = threadIdx.x >> 2, sub = threadIdx.x & 3;
                const uint64_t x = i < size ? list[i] : 0, w = i < size ? sm.pair_w[i] : 0;
                uint32_t larger = 0;
                uint64_t before = 0;
                for (uint32_t j = sub; j < size; j += 4) {
                    const bool l = list[j] > x;
                    larger += l;
                    before += l ? sm.pair_w[j] : 0;
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    larger += __shfl_xor_sync(0xffffffffu, larger, o);
                    before += __shfl_xor_sync(0xffffffffu, before, o);
                }
                if (by_k) {
                    if (i < size && larger == limit - 1) sm.found64[1] = before + w;
                    __syncthreads();
                    whole = sm.found64[1];
                }
                const uint64_t goal = by_p ? max((uint64_t)1, (uint64_t)ceil(p * (double)whole)) : ~0ull;
                before += above;
                const bool kept = i < size && larger < limit && before < goal;
                if (mode == kBin) {
                    if (kept && before + w >= goal) { sm.last_key = (uint32_t)(x >> 32); sm.last_index = (int)~(uint32_t)x; }
                } else {
                    const float v = key_value((uint32_t)(x >> 32));
                    const uint64_t kept_w = kept && sc.below(v) <= least ? w : 0;
                    __syncthreads();
                    if (sub == 0 && i < size) sm.pair_w[i] = kept_w;
                    __syncthreads();
                    uint64_t start = 0, total = 0;
                    for (uint32_t j = sub; j < size; j += 4) {
                        const uint64_t wj = sm.pair_w[j];
                        total += wj;
                        start += (uint32_t)list[j] > (uint32_t)x ? wj : 0;  // (~index: a lower index)
                    }
#pragma unroll
                    for (int o = 1; o < 4; o <<= 1) {
                        start += __shfl_xor_sync(0xffffffffu, start, o);
                        total += __shfl_xor_sync(0xffffffffu, total, o);
                    }
                    if (sub == 0 && falls_to(start, kept_w, u * (double)total, total)) choose((int)~(uint32_t)x, v, total);
                    return;
                }
            } else {
                // ---- longer: sorted
                sample_sort(list, (int)size);
                constexpr int PER = kSampleSort / kSampleThreads;
                const int each = ((int)size + kSampleThreads - 1) / kSampleThreads, at0 = (int)threadIdx.x * each;
                uint64_t w[PER], sum = 0;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const uint32_t i = at0 + j;
                    w[j] = j < each && i < limit ? sc.weight_of(key_value((uint32_t)(list[i] >> 32))) : 0;
                    sum += w[j];
                }
                uint64_t upto = above + block_upto64(sum, sm.sums) - sum;
                if (by_k) whole = sm.sums[kSampleWarps];
                // the first token at which the weight reaches the goal is the last one kept
                const uint64_t goal = by_p ? max((uint64_t)1, (uint64_t)ceil(p * (double)whole)) : ~0ull;
                if (threadIdx.x == 0) sm.found32[0] = limit - 1;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (w[j] > 0 && upto < goal && upto + w[j] >= goal) sm.found32[0] = at0 + j;  // (one thread)
                    upto += w[j];
                }
                __syncthreads();
                const uint32_t last = sm.found32[0];
                if (mode == kBin) {
                    if (threadIdx.x == 0) { sm.last_key = (uint32_t)(list[last] >> 32); sm.last_index = (int)~(uint32_t)list[last]; }
                } else {
                    // the choice: those kept in the order of their indices
                    int kept = 0;
                    for (uint32_t i = threadIdx.x; i <= last; i += kSampleThreads) kept += sc.below(key_value((uint32_t)(list[i] >> 32))) <= least;
                    uint32_t n;
                    block_scan(kept, sm.scan, &n);  // (min_p lets a beginning of the order through)
                    for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads) {
                        const uint64_t x = list[i];
                        list[i] = x << 32 | x >> 32;  // by ~index, descending: by index, ascending
                    }
                    __syncthreads();
                    sample_sort(list, (int)n);
                    const int some = ((int)n + kSampleThreads - 1) / kSampleThreads, at1 = (int)threadIdx.x * some;
                    sum = 0;
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        w[j] = j < some && at1 + j < (int)n ? sc.weight_of(key_value((uint32_t)list[at1 + j])) : 0;
                        sum += w[j];
                    }
                    upto = block_upto64(sum, sm.sums) - sum;
                    const uint64_t total = sm.sums[kSampleWarps];
                    const double target = u * (double)total;
                    bool done = false;
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        if (!done && falls_to(upto, w[j], target, total)) {
                            done = true;
                            const uint64_t x = list[at1 + j];
                            choose((int)~(uint32_t)(x >> 32), key_value((uint32_t)x), total);
                        }
                        upto += w[j];
                    }
                    return;
                }
            }
        }
        sync();
        const auto* first_cta = cluster.map_shared_rank(&sm, 0);
        last_key = first_cta->last_key;
        last_index = first_cta->last_index;
        if (rank > 0 && first_cta->listed != 0) {
            sync();
            return;
        }
    }

    // ---- the choice from the row
    auto weight_in = [&](float v, int i) -> uint64_t {
        const uint32_t key = order_key(v);
        const bool in = (key > last_key || (key == last_key && i <= last_index)) && sc.below(v) <= least;
        const uint64_t w = sc.weight_of(v);
        return in ? w : 0;
    };
    uint64_t mine = 0;
    if (mode == kAll && least == INFINITY) {
        sample_run<0>(row, run_lo, run_hi, [&](const float (&v)[E], int) {
#pragma unroll
            for (int e = 0; e < E; ++e) mine += sc.weight_of(v[e]);
        });
    } else {
        // (many pieces hold nothing that is kept; a little below what min_p asks for)
        const float from = fmaxf(mode == kBin ? key_value(last_key) : -INFINITY, sc.top - (float)least * 1.0001f - 1e-6f * fabsf(sc.top));
        sample_pieces<1>(row, run_lo, run_hi, [&](const uint4& raw, int at) {
            if (!(Logits<T>::largest(raw) >= from)) return;
            float v[E];
            Logits<T>::widen(raw, v);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (v[e] >= from) mine += weight_in(v[e], at + e);
        });
    }
    mine = warp_add64(mine);
    uint64_t start = __shfl_sync(0xffffffffu, block_upto64(lane == 0 ? mine : 0, sm.sums) - mine, 0);
    uint64_t total = sm.sums[kSampleWarps];
    if (ctas > 1) {
        if (threadIdx.x < ctas) cluster.map_shared_rank(&sm, threadIdx.x)->parts[rank] = total;
        cluster.sync();
        total = 0;
        for (int c = 0; c < ctas; ++c) {
            if (c < rank) start += sm.parts[c];
            total += sm.parts[c];
        }
    }
    const double target = u * (double)total;
    if (threadIdx.x == 0) sm.found32[0] = kSampleWarps;
    __syncthreads();
    if (lane == 0 && falls_to(start, mine, target, total)) { sm.found32[0] = warp; sm.found64[0] = start; }  // (one warp of the row)
    __syncthreads();
    if (sm.found32[0] == kSampleWarps) return;
    // its run again, a part for each warp of the CTA
    const int whose = (int)sm.found32[0], lo = min(row.pieces, (rank * kSampleWarps + whose) * per), hi = min(row.pieces, lo + per);
    const int each = (per / 32 + kSampleWarps - 1) / kSampleWarps * 32, part_lo = min(hi, lo + warp * each), part_hi = min(hi, part_lo + each);
    mine = 0;
    sample_run(row, part_lo, part_hi, [&](const float (&v)[E], int at) {
#pragma unroll
        for (int e = 0; e < E; ++e) mine += weight_in(v[e], at + e);
    });
    mine = warp_add64(mine);
    start = sm.found64[0] + __shfl_sync(0xffffffffu, block_upto64(lane == 0 ? mine : 0, sm.sums) - mine, 0);
    if (!falls_to(start, mine, target, total)) return;
    uint64_t sum = start;
    sample_run(row, part_lo, part_hi, [&](const float (&v)[E], int at) {
        uint64_t w[E], here = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) { w[e] = weight_in(v[e], at + e); here += w[e]; }
        const uint64_t upto = warp_upto64(here);
        uint64_t n = sum + upto - here;
        if (falls_to(n, here, target, total)) {  // (one lane, once)
            bool done = false;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (!done && falls_to(n, w[e], target, total)) {
                    done = true;
                    choose(at + e, v[e], total);
                }
                n += w[e];
            }
        }
        sum += __shfl_sync(0xffffffffu, upto, 31);
    });
}

}  // namespace msa
