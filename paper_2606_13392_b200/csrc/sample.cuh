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
constexpr int kSampleBins = 2048, kSampleList = 4096;
constexpr int kSampleSort = 1024;               // nuclei up to this are sorted, of larger ones only the bin they end in
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
        T v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at + e >= 0 && at + e < vocab ? __ldg(x + at + e) : T(-INFINITY);
        return *reinterpret_cast<const uint4*>(v);
    }
    static __device__ __forceinline__ uint4 nothing() {
        const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : (E == 8 && Logits<T>::HALF ? 0xFC00FC00u : 0xFF80FF80u);
        return make_uint4(w, w, w, w);
    }
};

// Pieces [lo, hi) of a warp: a run of the row, lanes side by side, four in flight.  f(piece, index of its first value) is called by
// all lanes of the warp (beyond the run: with -infinities).
template <class T, class F>
__device__ __forceinline__ void sample_pieces(const SampleRow<T>& row, int lo, int hi, F f) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 31;
    for (int p0 = lo; p0 < hi; p0 += 32 * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * 32 + lane;
            raw[u] = p < hi ? row.load(p) : SampleRow<T>::nothing();
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p0 + u * 32 < hi) f(raw[u], row.index(p0 + u * 32 + lane));
    }
}
// The same with the values as floats.
template <class T, class F>
__device__ __forceinline__ void sample_run(const SampleRow<T>& row, int lo, int hi, F f) {
    sample_pieces(row, lo, hi, [&](const uint4& raw, int at) {
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
        tct = (double)top * ct + kFront;
    }
    // Distance to the top (in 32 bits it would be rounded); a top of infinity comes with sample_slow only.
    __device__ __forceinline__ double below(float v) const { return (double)top - (double)v; }
    // 2^42 2^(-k/1024) 2^-r to the nearest whole number, `some` is false: 0.  2^(-k/1024) from a table and an exponent, 2^-r, |r| <=
    // 2^-10, by its Taylor series to the third power (off by less than 2^-46); the rounding by adding 2^52.
    __device__ __forceinline__ uint64_t power(int k, double r, bool some) const {
        constexpr double L = -0.69314718055994530942;
        const double p = fma(r, fma(r, fma(r, L * L * L / 6, L * L / 2), L), 1.0);
        const double w = table[k & (kSampleTable - 1)] * p;
        const double scaled = __hiloint2double(__double2hiint(w) + ((kSampleBits - (k >> 10)) << 20), __double2loint(w));
        const uint64_t whole = (uint64_t)__double_as_longlong(scaled + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
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
    // Bin of a logit, larger logits in lower bins; kSampleBins: its weight is 0.
    __device__ __forceinline__ int bin(float v) const {
        const float z = (top - v) * c32;
        return z < kSampleReach ? min((int)(z * (kSampleBins / kSampleReach)), kSampleBins - 1) : kSampleBins;
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
    uint32_t count[kSampleBins];
    union {
        struct { uint32_t lo[kSampleBins], hi[kSampleBins]; } mass;
        uint64_t list[kSampleList];    // (key, ~index): larger first means larger logit, then lower index
    };
    uint64_t sums[kSampleWarps + 1];
    uint32_t scan[33];
    float tops[kSampleWarps];
    // what a CTA tells the others (each is written once a row)
    struct { float top; int nan; } said;
    uint64_t total, above, part_total;
    uint32_t listed;
    // what the first CTA tells the others
    uint32_t last_key;
    int last_index;
    // results of a search by one thread
    uint64_t found64[2];
    uint32_t found32[3];
};

// Sorts list[0, n) in descending order (up to the next power of two, filled with zeros).
__device__ inline void sample_sort(uint64_t* list, int n) {
    int size = 32;
    while (size < n) size *= 2;
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

// The same for n <= kSampleThreads, a value a thread: thread i gets the i-th largest (0 from n on).  Partners of one warp trade
// places in registers.  `list` holds the values before; it is written on.
__device__ inline uint64_t sample_sort_short(uint64_t* list, int n) {
    const int i = threadIdx.x;
    int size = 32;
    while (size < n) size *= 2;
    uint64_t x = i < n ? list[i] : 0;
    if (size > 32) __syncthreads();
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            uint64_t y = 0;
            if (j >= 32) {
                if (i < size) list[i] = x;
                __syncthreads();
                if (i < size) y = list[i ^ j];
                __syncthreads();
            } else {
                y = __shfl_xor_sync(0xffffffffu, x, j);
            }
            const bool larger = ((i & k) == 0) == ((i & j) == 0);  // this thread keeps the larger of the two
            x = (x > y) == larger ? x : y;
        }
    }
    return x;
}

__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key); }

// ---------------------------------------------------------------- any row, by one CTA
// Whatever is kept, however many are equal: thresholds by the bits of the logits, 11, 11 and 10 at a time, each a pass over
// the row that adds up counts or weights of the digits; then the index among equal ones.  For rows that the lists below do not hold.
template <class T>
__device__ __noinline__ void sample_slow(const SampleArgs& a, int64_t row_number, const SampleRow<T>& row, const SampleScale& sc, double least, SampleSmem& sm,
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
    auto narrow = [&](bool by_mass, uint64_t target) {
        uint32_t prefix = 0;
        uint64_t want = target;
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
            for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) sm.count[i] = sm.mass.lo[i] = sm.mass.hi[i] = 0;
            __syncthreads();
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int at) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t k = order_key(v[e]);
                    if (!kept(v[e], at + e) || (round > 0 && k >> (shift + bits) != prefix)) continue;
                    const uint32_t bin = (k >> shift) & ((1u << bits) - 1);
                    atomicAdd(&sm.count[bin], 1u);
                    if (by_mass) {
                        const uint64_t w = weight_of(v[e]);
                        const uint32_t old = atomicAdd(&sm.mass.lo[bin], (uint32_t)w);
                        const uint32_t high = (uint32_t)(w >> 32) + (old + (uint32_t)w < old ? 1u : 0u);
                        if (high != 0) atomicAdd(&sm.mass.hi[bin], high);
                    }
                }
            });
            __syncthreads();
            uint64_t c[4], mine = 0;  // digits from the top, four a thread
            const int d = kSampleBins - 1 - 4 * (int)threadIdx.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = by_mass ? ((uint64_t)sm.mass.hi[d - j] << 32) + sm.mass.lo[d - j] : sm.count[d - j];
                mine += c[j];
            }
            uint64_t above = block_upto64(mine, sm.sums) - mine;
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
// A cluster of CTAs per row (one CTA where there are many rows), each with a run of it: a pass for the maximum; where something
// is filtered, a pass that counts the row in 2048 bins of equal width in log w, which the CTAs add up.
//   top_k: what is counted are the threads' own maxima, which the pass for the maximum has left: k of them are a bound that the k largest
//          reach, and hardly more.  (Every logit, where the threads are not many more than k.)  The tokens that reach it go to a
//          list in the first CTA, which sorts it, cuts it and chooses from it.
//   top_p alone: the counts bound the weight of each bin, and so the bins where the nucleus may end; a pass adds up the weights exactly,
//          of the row, and bin by bin between the bounds.  If the nucleus fits the list it is chosen from there; else only
//          the bin in which it ends is listed, to find its last token, and the choice is made as without filters:
//   no filters: every warp adds up its run, and the one that the target falls into finds the token.
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

    // 2^(-i/1024) from 2^(-i/32) and 2^(-i/1024) of the first 32
    if (threadIdx.x < 64) sm.root[threadIdx.x] = exp2((threadIdx.x < 32 ? (double)threadIdx.x / -32 : (double)(threadIdx.x - 32) / -1024));
    for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) sm.count[i] = sm.mass.lo[i] = sm.mass.hi[i] = 0;
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < kSampleTable; i += kSampleThreads) sm.table[i] = sm.root[i >> 5] * sm.root[32 + (i & 31)];

    // ---- the largest logit; this thread's own
    float own_top = -INFINITY, top;
    {
        sample_pieces(row, run_lo, run_hi, [&](const uint4& raw, int) { own_top = max_nan(own_top, Logits<T>::largest(raw)); });
        bool nan = __syncthreads_or(own_top != own_top) != 0;
        top = warp_max(own_top);
        if (lane == 0) sm.tops[warp] = top;
        __syncthreads();
        top = warp_max(sm.tops[lane % kSampleWarps]);
        if (ctas > 1) {
            if (threadIdx.x == 0) { sm.said.top = top; sm.said.nan = nan; }
            cluster.sync();
            const auto* other = cluster.map_shared_rank(&sm, lane % ctas);
            top = warp_max(other->said.top);
            nan = __any_sync(0xffffffffu, other->said.nan != 0);
        }
        nan |= !(temperature == temperature) || !(u == u);
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
    const double least = !greedy && min_p > 0.f ? fmax(0.0, -log((double)min_p) * T_) : INFINITY;
    const int k = greedy ? 1 : top_k;
    bool by_k = k > 0 && k < a.vocab;
    const bool by_p = !greedy && top_p < 1.f;

    // Adds up an array of all CTAs, everywhere: a part each, handed to the others.  (The arrays are the CTAs' own before.)
    auto merge = [&](uint32_t* lo, uint32_t* hi) {
        if (ctas == 1) { __syncthreads(); return; }
        cluster.sync();
        const int part = kSampleBins / ctas;
        for (int i = threadIdx.x; i < part; i += kSampleThreads) {
            const int at = rank * part + i;
            uint64_t sum = 0;
            for (int c = 0; c < ctas; ++c) {
                sum += *cluster.map_shared_rank(lo + at, c);
                if (hi) sum += (uint64_t)*cluster.map_shared_rank(hi + at, c) << 32;
            }
            for (int c = 0; c < ctas; ++c) {  // (nobody else reads or writes this part)
                *cluster.map_shared_rank(lo + at, c) = (uint32_t)sum;
                if (hi) *cluster.map_shared_rank(hi + at, c) = (uint32_t)(sum >> 32);
            }
        }
        cluster.sync();
    };

    enum { kAll, kList, kBin, kSlow };
    int mode = kAll, bin_lo = 0, bin_hi = kSampleBins;  // bins that are listed
    uint64_t whole = 0, above = 0;                      // weight of the row, of the bins before the listed ones
    constexpr int PER = kSampleBins / kSampleThreads;
    const int b0 = (int)threadIdx.x * PER;
    // the bin in which a count from the top reaches k: to found32[0], the count up to its end to found32[1]
    auto bin_of_count = [&](uint32_t* all) {
        uint32_t n[PER], mine = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) { n[j] = sm.count[b0 + j]; mine += n[j]; }
        uint32_t upto = block_scan(mine, sm.scan, all);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (upto < (uint32_t)k && upto + n[j] >= (uint32_t)k) { sm.found32[0] = b0 + j; sm.found32[1] = upto + n[j]; }  // (one thread)
            upto += n[j];
        }
        __syncthreads();
    };
    const bool tame = fabs(sc.tc) < 1048576.0;  // (weight_of; a top of infinity is not)
    // Twice as many threads as k, at least, or most of what they would list is not wanted.
    bool by_maxima = by_k && (int64_t)k * 2 <= (int64_t)ctas * kSampleThreads && tame;
    if (by_maxima) {
        const int b = sc.bin(own_top);
        if (b < kSampleBins) atomicAdd(&sm.count[b], 1u);
        merge(sm.count, nullptr);
        uint32_t all;
        bin_of_count(&all);
        by_maxima = all >= (uint32_t)k;
        if (by_maxima) {
            // (in units of the bins: what reaches the bin, not just the maxima)
            bin_hi = (int)sm.found32[0] + 1;
            mode = kList;
        } else {  // the threads' maxima are too few: count all
            for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) sm.count[i] = 0;
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
        merge(sm.count, nullptr);
        uint32_t all;
        bin_of_count(&all);
        by_k = by_k && (uint32_t)k < all;  // (the rest weighs nothing)
        if (by_k) {
            bin_hi = (int)sm.found32[0] + 1;
            mode = sm.found32[1] <= kSampleList ? kList : kSlow;
        } else if (by_p) {
            // Bounds of the weight up to each bin: a logit of bin b weighs 2^-(b+1)h to 2^-bh, h the width (and 10^-5 for the
            // 32-bit arithmetic of the bins).  The nucleus ends where the weight reaches top_p of the whole.
            uint32_t n[PER], counts = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) { n[j] = sm.count[b0 + j]; counts += n[j]; }
            const uint32_t before = block_scan(counts, sm.scan, &all);
            const double h = (double)kSampleReach / kSampleBins, p = (double)fmaxf(top_p, 0.f);
            double low = 0.0, low_of[PER], high_of[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const double w = (double)exp2f((float)(-(b0 + j) * h)) * n[j];
                high_of[j] = w * 1.00003;
                low_of[j] = w * 0.98555 * 0.99997;  // 2^-h
                low += low_of[j];
            }
            static_assert(kSampleTable == 1024 && kSampleBins == 2048, "the factor is 2^(-43/2048)");
            // (in whole numbers, for the scan: 2^-20 of the largest; rounded to the safe side below)
            const uint64_t lows = (uint64_t)(low * 1048576.0), low_upto = block_upto64(lows, sm.sums), low_all = sm.sums[kSampleWarps];
            double high = 0.0;
#pragma unroll
            for (int j = 0; j < PER; ++j) high += high_of[j];
            const uint64_t highs = (uint64_t)(high * 1048576.0) + 1, high_upto = block_upto64(highs, sm.sums), high_all = sm.sums[kSampleWarps];
            // first thread whose bins may hold the end, first whose bins certainly reach it
            const bool may = (double)high_upto >= p * (double)low_all, must = (double)low_upto >= p * (double)high_all;
            if (threadIdx.x == 0) { sm.found32[0] = 0; sm.found32[1] = kSampleBins; }
            __syncthreads();
            if (may && !((double)(high_upto - highs) >= p * (double)low_all)) sm.found32[0] = b0;
            if (must && !((double)(low_upto - lows) >= p * (double)high_all)) sm.found32[1] = b0 + PER;
            __syncthreads();
            const int from = (int)sm.found32[0], to = (int)sm.found32[1];
            // ---- exact weights: of the row, of the bins before `from`, of each bin in [from, to)
            uint64_t total = 0, earlier = 0;
            sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int b = sc.bin(v[e]);
                    if (b >= kSampleBins) continue;
                    const uint64_t w = sc.weight_of(v[e]);
                    total += w;
                    if (b < from) earlier += w;
                    else if (b < to) {
                        const uint32_t old = atomicAdd(&sm.mass.lo[b], (uint32_t)w);
                        const uint32_t up = (uint32_t)(w >> 32) + (old + (uint32_t)w < old ? 1u : 0u);
                        if (up != 0) atomicAdd(&sm.mass.hi[b], up);
                    }
                }
            });
            block_upto64(total, sm.sums);
            if (threadIdx.x == 0) sm.total = sm.sums[kSampleWarps];
            block_upto64(earlier, sm.sums);
            if (threadIdx.x == 0) sm.above = sm.sums[kSampleWarps];
            merge(sm.mass.lo, sm.mass.hi);
            for (int c = 0; c < ctas; ++c) {
                whole += *cluster.map_shared_rank(&sm.total, c);
                above += *cluster.map_shared_rank(&sm.above, c);
            }
            uint64_t m[PER], mass = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) { m[j] = ((uint64_t)sm.mass.hi[b0 + j] << 32) + sm.mass.lo[b0 + j]; mass += m[j]; }
            uint64_t upto = above + block_upto64(mass, sm.sums) - mass;
            const uint64_t goal = max((uint64_t)1, (uint64_t)ceil(p * (double)whole));
            uint32_t counted = before;
            if (threadIdx.x == 0) { sm.found32[0] = kSampleBins - 1; sm.found32[1] = 0xFFFFFFFFu; }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if (upto < goal && upto + m[j] >= goal && b0 + j >= from) {  // (one thread)
                    sm.found32[0] = b0 + j; sm.found32[1] = counted + n[j]; sm.found32[2] = n[j];
                    sm.found64[0] = upto;
                }
                upto += m[j];
                counted += n[j];
            }
            __syncthreads();
            bin_hi = (int)sm.found32[0] + 1;
            if (sm.found32[1] == 0xFFFFFFFFu) mode = kSlow;
            else if (sm.found32[1] <= kSampleSort) { mode = kList; above = 0; }
            else if (sm.found32[2] <= kSampleList) { mode = kBin; bin_lo = bin_hi - 1; above = sm.found64[0]; }
            else mode = kSlow;
        }
    }
    if (mode == kSlow) {
        if (ctas > 1) cluster.sync();  // (nobody reads the first CTA's memory any more)
        if (rank == 0) sample_slow<T>(a, r, row, sc, least, sm, greedy, top_k, top_p, T_, u);
        return;
    }

    if (mode != kAll) {
        // ---- the tokens of bins [bin_lo, bin_hi) into the first CTA's list, in any order
        if (ctas > 1) cluster.sync();  // (the list takes the place of the masses, which have been read)
        else __syncthreads();
        uint64_t *list = sm.list, *to = cluster.map_shared_rank(list, 0);
        uint32_t* listed = cluster.map_shared_rank(&sm.listed, 0);
        // (logits that reach the bins' lower end, or a little below: most pieces have none)
        const float least_listed = sc.top - (float)bin_hi * (kSampleReach / kSampleBins) / sc.c32 * 1.0001f - 1e-6f * fabsf(sc.top);
        sample_pieces(row, run_lo, run_hi, [&](const uint4& raw, int at) {
            if (!(Logits<T>::largest(raw) >= least_listed)) return;
            float v[E];
            Logits<T>::widen(raw, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int b = sc.bin(v[e]);
                if (b >= bin_lo && b < bin_hi) {
                    const uint32_t n = atomicAdd(listed, 1u);
                    if (n < kSampleList) to[n] = (uint64_t)order_key(v[e]) << 32 | (uint32_t)~(at + e);
                }
            }
        });
        if (ctas > 1) cluster.sync();
        else __syncthreads();
        const uint32_t size = *listed;
        if (ctas > 1 && mode == kBin) cluster.sync();  // (read by all before the first one goes on)
        if (mode == kList && rank > 0) return;  // (a bin's list is never too long: it was counted)
        if (size > kSampleList) {               // (more reach the bound than the list holds)
            sample_slow<T>(a, r, row, sc, least, sm, greedy, top_k, top_p, T_, u);
            return;
        }
        if (mode == kList && size <= kSampleThreads) {
            // ---- the choice from a short list: a token a thread
            const uint32_t i = threadIdx.x, limit = by_k ? min((uint32_t)k, size) : size;
            uint64_t x = sample_sort_short(list, (int)size);
            float v = key_value((uint32_t)(x >> 32));
            uint64_t w = i < limit ? sc.weight_of(v) : 0;
            uint64_t upto = block_upto64(w, sm.sums);
            if (by_k) whole = sm.sums[kSampleWarps];
            // kept: what comes before the goal is reached
            const uint64_t goal = by_p ? max((uint64_t)1, (uint64_t)ceil((double)fmaxf(top_p, 0.f) * (double)whole)) : ~0ull;
            const bool kept = i < limit && upto - w < goal && sc.below(v) <= least;
            const int n = __syncthreads_count(kept);  // (a beginning of the order)
            if (kept) list[i] = x << 32 | x >> 32;    // by ~index, descending: by index, ascending
            __syncthreads();
            x = sample_sort_short(list, n);
            v = key_value((uint32_t)x);
            w = i < (uint32_t)n ? sc.weight_of(v) : 0;
            upto = block_upto64(w, sm.sums);
            const uint64_t total = sm.sums[kSampleWarps];
            const double target = u * (double)total;
            // the first whose sum is beyond the target (where there is none: the last)
            if (w > 0 && ((double)upto > target || upto == total) && (double)(upto - w) <= target && upto - w < total) {
                a.token[r] = (int)~(uint32_t)(x >> 32);
                if (a.logprob) a.logprob[r] = greedy ? 0.f : (float)(-sc.below(v) / T_ - log((double)total / kSampleOne));
            }
            return;
        }
        if (rank == 0) {
            sample_sort(list, (int)size);
            constexpr int PER = kSampleList / kSampleThreads;
            const int per_thread = ((int)size + kSampleThreads - 1) / kSampleThreads, at0 = (int)threadIdx.x * per_thread;
            uint64_t w[PER], mine = 0;
            const uint32_t limit = by_k ? min((uint32_t)k, size) : size;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t i = at0 + j;
                w[j] = j < per_thread && i < limit ? sc.weight_of(key_value((uint32_t)(list[i] >> 32))) : 0;
                mine += w[j];
            }
            uint64_t upto = above + block_upto64(mine, sm.sums) - mine;
            if (by_k) whole = sm.sums[kSampleWarps];
            // the first token at which the weight reaches the goal is the last one kept
            const uint64_t goal = by_p ? max((uint64_t)1, (uint64_t)ceil((double)fmaxf(top_p, 0.f) * (double)whole)) : ~0ull;
            if (threadIdx.x == 0) sm.found32[0] = limit - 1;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if (w[j] > 0 && upto < goal && upto + w[j] >= goal) sm.found32[0] = at0 + j;  // (one thread)
                upto += w[j];
            }
            __syncthreads();
            const uint32_t last = sm.found32[0];
            if (threadIdx.x == 0) {
                sm.last_key = (uint32_t)(list[last] >> 32);
                sm.last_index = (int)~(uint32_t)list[last];
            }
            if (mode == kList) {
                // ---- the choice: those kept in the order of their indices
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
                const int each = ((int)n + kSampleThreads - 1) / kSampleThreads, from = (int)threadIdx.x * each;
                mine = 0;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    w[j] = j < each && from + j < (int)n ? sc.weight_of(key_value((uint32_t)list[from + j])) : 0;
                    mine += w[j];
                }
                upto = block_upto64(mine, sm.sums) - mine;
                const uint64_t total = sm.sums[kSampleWarps];
                const double target = u * (double)total;
                bool before_me = (double)upto > target || (upto == total && upto > 0);  // (chosen already)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    upto += w[j];
                    if (!before_me && w[j] > 0 && ((double)upto > target || upto == total)) {
                        before_me = true;
                        const uint64_t x = list[from + j];
                        a.token[r] = (int)~(uint32_t)(x >> 32);
                        if (a.logprob)
                            a.logprob[r] = greedy ? 0.f : (float)(-sc.below(key_value((uint32_t)x)) / T_ - log((double)total / kSampleOne));
                    }
                }
                return;
            }
        }
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    }

    // ---- the choice from the row
    const uint32_t last_key = mode == kBin ? *cluster.map_shared_rank(&sm.last_key, 0) : 0u;
    const int last_index = mode == kBin ? *cluster.map_shared_rank(&sm.last_index, 0) : a.vocab;
    auto weight_in = [&](float v, int i) -> uint64_t {
        const uint32_t key = order_key(v);
        if (key < last_key || (key == last_key && i > last_index)) return 0;
        const double d = sc.below(v);
        return d <= least ? sc.weight(d) : 0;
    };
    uint64_t mine = 0;
    if (mode == kAll && least == INFINITY) {
        sample_run(row, run_lo, run_hi, [&](const float (&v)[E], int) {
#pragma unroll
            for (int e = 0; e < E; ++e) mine += sc.weight_of(v[e]);
        });
    } else {
        // (most pieces hold nothing that is kept; a little below what min_p asks for)
        const float from = fmaxf(mode == kBin ? key_value(last_key) : -INFINITY, sc.top - (float)least * 1.0001f - 1e-6f * fabsf(sc.top));
        sample_pieces(row, run_lo, run_hi, [&](const uint4& raw, int at) {
            if (!(Logits<T>::largest(raw) >= from)) return;
            float v[E];
            Logits<T>::widen(raw, v);
#pragma unroll
            for (int e = 0; e < E; ++e) mine += weight_in(v[e], at + e);
        });
    }
    mine = warp_add64(mine);
    uint64_t start = __shfl_sync(0xffffffffu, block_upto64(lane == 0 ? mine : 0, sm.sums) - mine, 0);
    uint64_t total = sm.sums[kSampleWarps], cta_start = 0;
    if (ctas > 1) {
        if (threadIdx.x == 0) sm.part_total = total;
        cluster.sync();
        total = 0;
        for (int c = 0; c < ctas; ++c) {
            const uint64_t x = *cluster.map_shared_rank(&sm.part_total, c);
            if (c < rank) cta_start += x;
            total += x;
        }
        start += cta_start;
    }
    const double target = u * (double)total;
    // Does the choice fall to weights [from, from + n)?  (The last kept token, where rounding or a u of 1 or more leaves none.)
    auto falls_to = [&](uint64_t from, uint64_t n) {
        return n > 0 && ((double)(from + n) > target || from + n == total) && ((double)from <= target || from == 0);
    };
    if (threadIdx.x == 0) sm.found32[0] = kSampleWarps;
    __syncthreads();
    if (lane == 0 && falls_to(start, mine)) { sm.found32[0] = warp; sm.found64[0] = start; }  // (one warp of the row)
    __syncthreads();
    if (sm.found32[0] < kSampleWarps) {
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
        if (falls_to(start, mine)) {
            uint64_t sum = start;
            sample_run(row, part_lo, part_hi, [&](const float (&v)[E], int at) {
                uint64_t w[E], here = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) { w[e] = weight_in(v[e], at + e); here += w[e]; }
                const uint64_t upto = warp_upto64(here);
                uint64_t n = sum + upto - here;
                if (falls_to(n, here)) {  // (one lane, once)
                    bool chosen = false;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (!chosen && falls_to(n, w[e])) {
                            chosen = true;
                            a.token[r] = at + e;
                            if (a.logprob) a.logprob[r] = (float)(-sc.below(v[e]) / T_ - log((double)total / kSampleOne));
                        }
                        n += w[e];
                    }
                }
                sum += __shfl_sync(0xffffffffu, upto, 31);
            });
        }
    }
    if (ctas > 1) cluster.sync();  // (the others may still read this CTA's sum)
}

}  // namespace msa
