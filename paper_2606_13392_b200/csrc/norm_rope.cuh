// Norms of queries and keys for each head with the position rotation in the same pass, their gradients, and the
// append of keys and values to a paged cache with both applied on the way.
//
//   n = x rsqrt(mean(x^2) + eps) w      (one mean per head; w = none: n = x)
//   y = rotation of the pairs of n's first `rot` elements by the angle p f_i, times mscale; the rest unchanged
//
// Bound by HBM (about 2 flop per byte), so the design is about bytes in flight and about doing the per-token work
// once.  A head is 16 bytes for each of d/8 lanes (a power of two reserved: 8, 16 or 32); a warp of the forward kernel
// loads four heads per lane group before it computes.  Both outputs of a pair need both inputs: in the half layout the partner sits rot/16 lanes away and its raw bf16 come by shuffle (four registers
// for eight elements), in the interleaved layout it is in the same register.
// Angles are formed in 64 bits as turns, p (f / 2 pi) minus the nearest whole
// number, because a 32-bit angle at position 10^6 is off by 0.03 rad; sine and cosine of the remainder are 32-bit.
// The forward kernel's CTAs compute them once per (token, pair) into shared memory, as coefficients of the partner form
//   y_e = rstd (x_e A_e + x_partner B_e),   A_e = w_e cos, B_e = -+ w_partner sin
// which holds for the elements behind `rot` too (A = w, B = 0).
// Sums of squares and all products are 32-bit; the one rounding is the store (bf16, or E4M3 saturating).
#pragma once

#include <type_traits>

#include "common.cuh"

namespace msa {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kRopeMaxTile = 32;  // tokens a CTA prepares at a time

// Shared memory of a token's coefficients: two sets of 16 floats a lane.  A launch gets 48 KB, the positions and places of
// the tile's tokens included; more would have to be asked for and would cost the CTAs side by side that hide latencies.
constexpr int rope_token_bytes(int lanes_per_head) { return 2 * lanes_per_head * 16 * (int)sizeof(float); }
constexpr int rope_tile_limit(int lanes_per_head) { return kRopeMaxTile * 8 / lanes_per_head; }
constexpr int kRopeStaticBytes = kRopeMaxTile * 2 * (int)sizeof(int64_t);
static_assert(rope_tile_limit(8) * rope_token_bytes(8) + kRopeStaticBytes <= 48 * 1024 &&
              rope_tile_limit(16) * rope_token_bytes(16) + kRopeStaticBytes <= 48 * 1024 &&
              rope_tile_limit(32) * rope_token_bytes(32) + kRopeStaticBytes <= 48 * 1024, "shared memory of a launch");

struct RopeArgs {
    const double* freqs;  // [rot/2] radians per position, or null (no rotation)
    int rot, interleaved;
    float mscale;
};

// One set of heads: rows of n_heads*d bf16 at x + token*stride; w: weights of its norm or null.
struct RopeHeads {
    const __nv_bfloat16* x;
    int64_t stride;
    int n_heads;
    const void* w;
    __nv_bfloat16* out;  // rows of n_heads*d, dense
};

// The paged cache as the kernels see it.
struct PagedView {
    const int32_t* cu_q;     // [batch+1] first new token of each sequence
    const int32_t* kv_lens;  // [batch]   tokens of each sequence, the new ones included
    const int32_t* table;    // [batch, max_pages] page of each run of page_size tokens
    int batch, max_pages, n_pages, page_size, H_kv;
};

__device__ __forceinline__ float weight_at(const void* w, int c, bool w32) {
    return w32 ? static_cast<const float*>(w)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c]);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight bf16 as four pairs of floats, and back: packed two-float arithmetic halves the instructions, which is what
// bounds these kernels next to the bytes.
struct F8v { float2 v[4]; };
__device__ __forceinline__ F8v widen8(const uint4& u) {
    return F8v{{bf16x2_to_float2(u.x), bf16x2_to_float2(u.y), bf16x2_to_float2(u.z), bf16x2_to_float2(u.w)}};
}
__device__ __forceinline__ uint4 narrow8(const F8v& f) {
    return make_uint4(pack2(f.v[0].x, f.v[0].y), pack2(f.v[1].x, f.v[1].y), pack2(f.v[2].x, f.v[2].y), pack2(f.v[3].x, f.v[3].y));
}
__device__ __forceinline__ uint2 narrow8_e4m3(const F8v& f) {  // nearest, beyond the range the largest
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __nv_cvt_float2_to_fp8x2(f.v[i], __NV_SATFINITE, __NV_E4M3);
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
__device__ __forceinline__ F8v load8(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    return F8v{{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}
__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }

template <int LPH>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The partners of a lane's eight elements: other lane (half layout), swapped neighbours (interleaved), zero where
// the head is not rotated.
__device__ __forceinline__ uint4 rope_partner(const uint4& v, int partner_lane, bool turned, bool interleaved) {
    uint4 p;
    if (interleaved) {
        p = make_uint4(__funnelshift_l(v.x, v.x, 16), __funnelshift_l(v.y, v.y, 16), __funnelshift_l(v.z, v.z, 16),
                       __funnelshift_l(v.w, v.w, 16));
    } else {
        p.x = __shfl_sync(0xffffffffu, v.x, partner_lane); p.y = __shfl_sync(0xffffffffu, v.y, partner_lane);
        p.z = __shfl_sync(0xffffffffu, v.z, partner_lane); p.w = __shfl_sync(0xffffffffu, v.w, partner_lane);
    }
    return turned ? p : make_uint4(0u, 0u, 0u, 0u);
}

// cos and sin (times mscale) of pair i at position pos.
__device__ __forceinline__ void rope_angle(const RopeArgs& rp, int64_t pos, int i, float& c, float& s) {
    const double turns = (double)pos * (rp.freqs[i] * 0.15915494309189535);
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    c *= rp.mscale; s *= rp.mscale;
}

// Elements of pair i.
__device__ __forceinline__ int rope_first(const RopeArgs& rp, int i) { return rp.interleaved ? 2 * i : i; }
__device__ __forceinline__ int rope_second(const RopeArgs& rp, int i) { return rp.interleaved ? 2 * i + 1 : i + rp.rot / 2; }

// Sequence of new token i: the last s with cu_q[s] <= i, by a 32-way search of one warp.  -1 behind the last
// sequence.  (Empty sequences share their start with the next one and are passed over.)
__device__ __forceinline__ int paged_seq_of(const PagedView& c, int i) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = c.batch;  // cu_q[lo] <= i; cu_q[hi] > i
    if (c.batch == 0 || i >= c.cu_q[c.batch] || i < c.cu_q[0]) return -1;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = min(lo + (lane + 1) * step, hi);  // lane 31 reaches hi
        const unsigned above = __ballot_sync(0xffffffffu, at >= hi || c.cu_q[at] > i);
        const int first = __ffs(above) - 1;              // first probe whose start is beyond i
        hi = min(lo + (first + 1) * step, hi);
        lo = lo + first * step;
    }
    return lo;
}

// Measured: 32768 tokens of 64 + 8 heads of 128 in 204 - 227 us, 83 - 92 % of the copy bandwidth (boards and surroundings
// differ); 8 + 1 heads of 128 in 53 us, 44 %, of 256 (16384 tokens) in 43 us, 54 %; 32 tokens of 64 + 8 heads in 4 us.
// (Warps on their own with asynchronous copies, the gradient kernel's form, were slower here: 250 against 212 us for 32768
// tokens of 64 + 8 heads.  One reduction and half the bytes per output leave the independent heads of an item enough.)
// Forward (APPEND = false: q and k to q.out and k.out; true: k and v to the cache, q to q.out).
// Coefficients in shared memory: [token][set 0 = q, 1 = k][lane of the head][A 0..7, B 0..7].
// EXACT: a head fills its lanes (d = 8 LPH).
template <int LPH, bool EXACT, bool APPEND, bool F8>
__global__ void __launch_bounds__(kRopeThreads)
norm_rope_kernel(RopeArgs rp, RopeHeads q, RopeHeads k, RopeHeads v, int64_t n_tokens, int d_arg, float eps, bool w32,
                 const int64_t* __restrict__ positions, int tile, int heads_per_cta, PagedView cache,
                 void* __restrict__ k_pool, void* __restrict__ v_pool, int* status) {
    constexpr int HPW = 32 / LPH;                // heads a warp holds side by side
    constexpr int U = 4;                         // heads per lane in flight
    extern __shared__ __align__(16) float coef[];  // [tile][2][LPH][16]
    __shared__ int64_t s_pos[kRopeMaxTile], s_row[kRopeMaxTile];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = lane % LPH, sub = lane / LPH;
    const int d = EXACT ? LPH * 8 : d_arg;
    const float inv_d = 1.0f / (float)d;
    const bool active = EXACT || j * 8 < d;
    const int half = rp.rot / 2;
    const bool turned = rp.freqs != nullptr && j * 8 < rp.rot;
    const int partner = sub * LPH + (j * 8 < half ? j + half / 8 : j - half / 8);
    // items of a token: runs of U*HPW heads of q, then of k, then of v
    const int run = U * HPW;
    const int n_q = (q.n_heads + run - 1) / run, n_k = (k.n_heads + run - 1) / run;
    const int n_all = n_q + n_k + (APPEND ? (v.n_heads + run - 1) / run : 0);
    const int item_lo = blockIdx.y * heads_per_cta;  // (in items)
    const int item_n = min(heads_per_cta, n_all - item_lo);

    for (int64_t t0 = (int64_t)blockIdx.x * tile; t0 < n_tokens; t0 += (int64_t)gridDim.x * tile) {
        const int nt = (int)min((int64_t)tile, n_tokens - t0);
        if constexpr (APPEND) {
            for (int t = warp; t < nt; t += kRopeWarps) {
                const int i = (int)(t0 + t);
                const int s = paged_seq_of(cache, i);
                if (lane == 0) {
                    int64_t pos = 0, row = -2;  // -2: behind the last sequence; -1: no place in the cache
                    if (s >= 0) {
                        const int end = cache.cu_q[s + 1];
                        pos = (int64_t)cache.kv_lens[s] - (end - i);
                        row = -1;
                        if (pos >= 0 && pos / cache.page_size < cache.max_pages) {
                            const int page = cache.table[(int64_t)s * cache.max_pages + pos / cache.page_size];
                            if (page >= 0 && page < cache.n_pages)
                                row = (int64_t)page * cache.page_size + pos % cache.page_size;
                        }
                        if (row < 0) report_async(status, kAsyncBadIndex, 0x501);
                    }
                    s_pos[t] = pos; s_row[t] = row;
                }
            }
        } else if (threadIdx.x < nt) {
            s_pos[threadIdx.x] = positions != nullptr ? positions[t0 + threadIdx.x] : 0;
        }
        __syncthreads();
        // coefficients: the rotated pairs, then the elements that stay
        if (rp.freqs != nullptr)
            for (int e = threadIdx.x; e < nt * half; e += kRopeThreads) {
                const int t = e / half, i = e - t * half;
                float c, s;
                rope_angle(rp, s_pos[t], i, c, s);
                const int a = rope_first(rp, i), b = rope_second(rp, i);
#pragma unroll
                for (int set = 0; set < 2; ++set) {
                    const void* w = set == 0 ? q.w : k.w;
                    const float wa = w != nullptr ? weight_at(w, a, w32) : 1.f, wb = w != nullptr ? weight_at(w, b, w32) : 1.f;
                    float* to = coef + (t * 2 + set) * (LPH * 16);
                    to[(a >> 3) * 16 + (a & 7)] = wa * c;
                    to[(a >> 3) * 16 + 8 + (a & 7)] = -wb * s;
                    to[(b >> 3) * 16 + (b & 7)] = wb * c;
                    to[(b >> 3) * 16 + 8 + (b & 7)] = wa * s;
                }
            }
        const int first_plain = rp.freqs != nullptr ? rp.rot : 0;
        for (int e = threadIdx.x; e < nt * (d - first_plain); e += kRopeThreads) {
            const int t = e / (d - first_plain), c = first_plain + e - t * (d - first_plain);
#pragma unroll
            for (int set = 0; set < 2; ++set) {
                const void* w = set == 0 ? q.w : k.w;
                float* to = coef + (t * 2 + set) * (LPH * 16) + (c >> 3) * 16 + (c & 7);
                to[0] = w != nullptr ? weight_at(w, c, w32) : 1.f;
                to[8] = 0.f;
            }
        }
        __syncthreads();
        // One item: U loads per lane group in flight, then head after head.
        auto heads = [&](const RopeHeads& hs, auto set_c, int t, int item, void* to, int64_t to_row) {
            constexpr int set = decltype(set_c)::value;
            const int h0 = item * run + sub, left = hs.n_heads - item * run;  // this lane group's first head; heads of the item
            const __nv_bfloat16* src = hs.x + (t0 + t) * hs.stride + (int64_t)h0 * d + j * 8;
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u] = make_uint4(0u, 0u, 0u, 0u);
                if (active && (left >= run || h0 + u * HPW < hs.n_heads)) x[u] = *reinterpret_cast<const uint4*>(src + u * HPW * d);
            }
            F8v A, B;
            if constexpr (set < 2) {
                const float* from = coef + (t * 2 + set) * (LPH * 16) + j * 16;
                A = load8(from);
                B = load8(from + 8);
            }
            const int64_t at0 = (to_row * hs.n_heads + h0) * d + j * 8;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (left < run && u * HPW >= left) break;  // (the same for the whole warp)
                F8v y = widen8(x[u]);
                if constexpr (set < 2) {
                    float2 r = twice(1.f);
                    if (hs.w != nullptr) {
                        float2 ss = __fmul2_rn(y.v[0], y.v[0]);
#pragma unroll
                        for (int e = 1; e < 4; ++e) ss = __ffma2_rn(y.v[e], y.v[e], ss);
                        r = twice(rsqrtf(fmaf(group_sum<LPH>(ss.x + ss.y), inv_d, eps)));
                    }
                    const F8v p = widen8(rope_partner(x[u], partner, turned, rp.interleaved));
#pragma unroll
                    for (int e = 0; e < 4; ++e) y.v[e] = __fmul2_rn(r, __ffma2_rn(y.v[e], A.v[e], __fmul2_rn(p.v[e], B.v[e])));
                }
                if (!active || (left < run && h0 + u * HPW >= hs.n_heads)) continue;
                const int64_t at = at0 + u * HPW * d;
                if constexpr (F8 && set > 0) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(to) + at) = narrow8_e4m3(y);
                else *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(to) + at) = narrow8(y);
            }
        };
        for (int it = warp; it < nt * item_n; it += kRopeWarps) {
            const int t = it / item_n;
            const int item = item_lo + it - t * item_n;
            const int64_t row = APPEND ? s_row[t] : t0 + t;
            if (item < n_q) {
                if (row != -2) heads(q, std::integral_constant<int, 0>{}, t, item, q.out, t0 + t);
            } else if (row < 0) {
                continue;
            } else if (item < n_q + n_k) {
                heads(k, std::integral_constant<int, 1>{}, t, item - n_q, APPEND ? k_pool : k.out, row);
            } else if constexpr (APPEND) {
                heads(v, std::integral_constant<int, 2>{}, t, item - n_q - n_k, v_pool, row);
            }
        }
        __syncthreads();
    }
}

// 16 bytes to shared memory without registers or waiting.
__device__ __forceinline__ void copy16_async(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }


// Gradients.  With g = (the transposed rotation of dy) and xh = x rstd:
//   dw = sum over tokens and heads of g xh,   dx = rstd (g w - xh mean(g w xh))      (w = none: dx = g)
// rstd is computed again from x: that is cheaper than keeping it.  Two tensors in, one out, and two reductions per head:
// what it takes is bytes in flight, and registers do not hold enough of them.  So warps work alone, without CTA barriers:
// a step is the heads that fit a warp side by side, and every warp takes an equal run of the steps of all tokens; it
// computes a token's angles into a table of its own, and its lanes copy their 16 bytes of x and dy of the next
// kGradStages - 1 steps to shared memory asynchronously (each lane reads back only what it copied).  The first q_ctas
// CTAs do the queries, the others the keys (one set of weights and sums in registers).  A lane accumulates its eight elements of dw over all its steps; lanes and warps of a CTA join in
// a fixed order, CTAs leave a row each in the workspace and norm_rope_dw_kernel adds the rows in order, so equal calls
// give equal bits.
// Measured: 8192 tokens of 64 + 4 heads of 128 in 85 - 92 us, 72 - 78 % of the copy bandwidth, issue slots 65 % busy
// (two heads per lane group in registers and CTA barriers: 117 us).
// Table: [lane of the head][cos 0..7, signed sin 0..7].
constexpr int kGradThreads = 128, kGradWarps = kGradThreads / 32;
constexpr int kGradCtas = 4;    // per SM
constexpr int kGradStages = 4;  // steps of 32 lanes x 16 bytes of x and of dy
struct RopeGrads {
    const __nv_bfloat16* dy;  // rows of n_heads*d, at dy + token*stride
    int64_t stride;
    __nv_bfloat16* dx;        // dense
};

template <int LPH>
constexpr size_t grad_smem() {
    return (size_t)kGradWarps * (kGradStages * 2 * 32 * sizeof(uint4) + LPH * 16 * sizeof(float));
}

template <int LPH, bool EXACT>
__global__ void __launch_bounds__(kGradThreads, kGradCtas)
norm_rope_grad_kernel(RopeArgs rp, RopeHeads q, RopeHeads k, RopeGrads gq, RopeGrads gk, int64_t n_tokens, int d_arg,
                      float eps, bool w32, const int64_t* __restrict__ positions, int q_ctas,
                      float* __restrict__ dw_rows) {
    constexpr int HPW = 32 / LPH;  // heads of a step, side by side
    extern __shared__ __align__(16) uint8_t grad_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* ring = reinterpret_cast<uint4*>(grad_raw) + warp * (kGradStages * 64) + lane;  // [stage][x, dy][lane]
    float* table = reinterpret_cast<float*>(grad_raw + (size_t)kGradWarps * kGradStages * 64 * sizeof(uint4)) + warp * (LPH * 16);
    const bool is_k = (int)blockIdx.x >= q_ctas;
    const RopeHeads& hs = is_k ? k : q;
    const RopeGrads& gs = is_k ? gk : gq;
    const int64_t mine = (is_k ? blockIdx.x - q_ctas : blockIdx.x) * kGradWarps + warp;  // of `warps`
    const int64_t warps = (is_k ? gridDim.x - q_ctas : q_ctas) * kGradWarps;
    const int j = lane % LPH, sub = lane / LPH;
    const int d = EXACT ? LPH * 8 : d_arg;
    const float inv_d = 1.0f / (float)d;
    const bool active = EXACT || j * 8 < d;
    const int half = rp.rot / 2;
    const bool turned = rp.freqs != nullptr && j * 8 < rp.rot;
    const int partner = sub * LPH + (j * 8 < half ? j + half / 8 : j - half / 8);
    const bool norm = hs.w != nullptr;
    const int first_plain = rp.freqs != nullptr ? rp.rot : 0;
    const int groups = (hs.n_heads + HPW - 1) / HPW;  // steps of a token
    const int64_t steps = n_tokens * groups, lo = steps / warps * mine + min(mine, steps % warps);
    int64_t left = steps / warps + (mine < steps % warps);
    F8v w, dw;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        w.v[e] = active && norm ? make_float2(weight_at(hs.w, j * 8 + 2 * e, w32), weight_at(hs.w, j * 8 + 2 * e + 1, w32)) : twice(1.f);
        dw.v[e] = twice(0.f);
    }
    int64_t t = groups > 0 ? lo / groups : 0;
    int g0 = (int)(lo - t * groups);
    // the copies' place in the run, kGradStages - 1 steps ahead
    int64_t ahead = left, ahead_t = t;
    int ahead_g = g0, put = 0;
    auto copy_next = [&]() {
        if (ahead > 0) {
            const int h = ahead_g * HPW + sub;
            if (active && h < hs.n_heads) {
                const int64_t at = (int64_t)h * d + j * 8;
                if (norm) copy16_async(ring + put * 64, hs.x + ahead_t * hs.stride + at);
                copy16_async(ring + put * 64 + 32, gs.dy + ahead_t * gs.stride + at);
            }
            --ahead;
            if (++ahead_g == groups) { ahead_g = 0; ++ahead_t; }
        }
        put = put + 1 == kGradStages ? 0 : put + 1;
        copy_async_commit();  // (an empty group at the end keeps the count)
    };
    for (int i = 0; i < kGradStages - 1; ++i) copy_next();
    int get = 0;
    for (; left > 0; ++t, g0 = 0) {
        const int g_hi = (int)min((int64_t)groups, g0 + left);
        left -= g_hi - g0;
        const int64_t pos = positions != nullptr ? positions[t] : 0;
        __syncwarp();
        if (rp.freqs != nullptr)
            for (int i = lane; i < half; i += 32) {
                float c, s;
                rope_angle(rp, pos, i, c, s);
                const int a = rope_first(rp, i), b = rope_second(rp, i);
                table[(a >> 3) * 16 + (a & 7)] = c;
                table[(a >> 3) * 16 + 8 + (a & 7)] = s;
                table[(b >> 3) * 16 + (b & 7)] = c;
                table[(b >> 3) * 16 + 8 + (b & 7)] = -s;
            }
        for (int c = first_plain + lane; c < LPH * 8; c += 32) {
            table[(c >> 3) * 16 + (c & 7)] = c < d ? 1.f : 0.f;  // (lanes without elements add zeros to the sums)
            table[(c >> 3) * 16 + 8 + (c & 7)] = 0.f;
        }
        __syncwarp();
        const F8v c = load8(table + j * 16), s = load8(table + j * 16 + 8);
        __nv_bfloat16* to = gs.dx + (t * hs.n_heads + g0 * HPW + sub) * d + j * 8;
        for (int gi = g0; gi < g_hi; ++gi, to += HPW * d) {
            copy_async_wait<kGradStages - 2>();
            const bool here = active && gi * HPW + sub < hs.n_heads;
            const uint4 none = make_uint4(0u, 0u, 0u, 0u);
            const uint4 xv = here && norm ? ring[get * 64] : none, gv = here ? ring[get * 64 + 32] : none;
            get = get + 1 == kGradStages ? 0 : get + 1;
            copy_next();
            F8v g = widen8(gv);
            const F8v gp = widen8(rope_partner(gv, partner, turned, rp.interleaved));
#pragma unroll
            for (int e = 0; e < 4; ++e) g.v[e] = __ffma2_rn(g.v[e], c.v[e], __fmul2_rn(gp.v[e], s.v[e]));
            if (norm) {
                const F8v x = widen8(xv);
                F8v gw;
                float2 ss = twice(0.f), dot = twice(0.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    gw.v[e] = __fmul2_rn(g.v[e], w.v[e]);
                    ss = __ffma2_rn(x.v[e], x.v[e], ss);
                    dot = __ffma2_rn(gw.v[e], x.v[e], dot);
                }
                const float sum = group_sum<LPH>(ss.x + ss.y), prod = group_sum<LPH>(dot.x + dot.y);
                const float r = rsqrtf(fmaf(sum, inv_d, eps));
                const float m = -(prod * inv_d * r * r);  // times x = -xh mean(g w xh)
                // (an absent head adds nothing; with eps = 0 its r is infinite)
                const float2 r2 = twice(r), m2 = twice(m), rd = twice(here ? r : 0.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dw.v[e] = __ffma2_rn(g.v[e], __fmul2_rn(x.v[e], rd), dw.v[e]);
                    g.v[e] = __fmul2_rn(r2, __ffma2_rn(x.v[e], m2, gw.v[e]));
                }
            }
            if (here) *reinterpret_cast<uint4*>(to) = narrow8(g);
        }
    }
    copy_async_wait<0>();
    if (dw_rows == nullptr) return;
    __syncthreads();
    float* join = reinterpret_cast<float*>(grad_raw);  // [warp][LPH * 8]
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float sum = e & 1 ? dw.v[e >> 1].y : dw.v[e >> 1].x;
#pragma unroll
        for (int o = 16; o >= LPH; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (sub == 0) join[warp * (LPH * 8) + j * 8 + e] = sum;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += kGradThreads) {
        float sum = 0.f;
        for (int i = 0; i < kGradWarps; ++i) sum += join[i * (LPH * 8) + c];
        dw_rows[(int64_t)blockIdx.x * d + c] = sum;
    }
}

// dw[c] = sum over the rows of the q CTAs (blockIdx.y = 0) or the k CTAs, 32 columns per CTA: 32 x 32 threads, each row
// class in order, then a tree.
__global__ void __launch_bounds__(1024)
norm_rope_dw_kernel(const float* __restrict__ rows, int q_rows, int n_rows, int d, float* __restrict__ dwq, float* __restrict__ dwk) {
    __shared__ float s[32][33];
    float* to = blockIdx.y == 0 ? dwq : dwk;
    if (to == nullptr) return;
    const int first = blockIdx.y == 0 ? 0 : q_rows, last = blockIdx.y == 0 ? q_rows : n_rows;
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x >> 5;
    float sum = 0.f;
    if (c < d)
        for (int r = first + r0; r < last; r += 32) sum += rows[(int64_t)r * d + c];
    s[r0][threadIdx.x & 31] = sum;
    __syncthreads();
    const float total = warp_sum(s[threadIdx.x & 31][r0]);  // warp r0 owns column r0 of the 32
    const int col = blockIdx.x * 32 + r0;
    if ((threadIdx.x & 31) == 0 && col < d) to[col] = total;
}

}  // namespace msa
