// Norms of queries and keys for each head with the position rotation in the same pass, their gradients, and the
// append of keys and values to a paged cache with both applied on the way.
//
//   n = x rsqrt(mean(x^2) + eps) w      (one mean per head; w = none: n = x)
//   y = rotation of the pairs of n's first `rot` elements by the angle p f_i, times mscale; the rest unchanged
//
// Bound by HBM (about 2 flop per byte), so the design is about bytes in flight and about doing the per-token work
// once.  A head is 16 bytes for each of d/8 lanes (a power of two reserved: 8, 16 or 32), a warp loads U heads per
// lane group before it computes.  Both outputs of a pair need both inputs: in the half layout the partner sits
// rot/16 lanes away and its raw bf16 come by shuffle (four registers for eight elements), in the interleaved
// layout it is in the same register.  Angles are formed in 64 bits as turns, p (f / 2 pi) minus the nearest whole
// number, because a 32-bit angle at position 10^6 is off by 0.03 rad; sine and cosine of the remainder are 32-bit.
// A CTA computes them once per (token, pair) into shared memory, as coefficients of the partner form
//   y_e = rstd (x_e A_e + x_partner B_e),   A_e = w_e cos, B_e = -+ w_partner sin
// which holds for the elements behind `rot` too (A = w, B = 0).
// Sums of squares and all products are 32-bit; the one rounding is the store (bf16, or E4M3 saturating).
#pragma once

#include <type_traits>

#include "common.cuh"

namespace msa {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kRopeMaxTile = 8;  // tokens a CTA prepares at a time

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

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    const float2 a = bf16x2_to_float2(v.x), b = bf16x2_to_float2(v.y), c = bf16x2_to_float2(v.z), d = bf16x2_to_float2(v.w);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// Eight floats -> eight E4M3 (nearest, beyond the range the largest).
__device__ __forceinline__ uint2 pack8_e4m3(const float (&f)[8]) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i], f[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

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

// Forward (APPEND = false: q and k to q.out and k.out; true: k and v to the cache, q to q.out).
// Coefficients in shared memory: [token][set 0 = q, 1 = k][lane of the head][A 0..7, B 0..7].
template <int LPH, bool APPEND, bool F8>
__global__ void __launch_bounds__(kRopeThreads)
norm_rope_kernel(RopeArgs rp, RopeHeads q, RopeHeads k, RopeHeads v, int64_t n_tokens, int d, float eps, bool w32,
                 const int64_t* __restrict__ positions, int tile, int heads_per_cta, PagedView cache,
                 void* __restrict__ k_pool, void* __restrict__ v_pool, int* status) {
    constexpr int HPW = 32 / LPH;                // heads a warp holds side by side
    constexpr int U = 4;                         // heads per lane in flight
    extern __shared__ __align__(16) float coef[];  // [tile][2][LPH][16]
    __shared__ int64_t s_pos[kRopeMaxTile], s_row[kRopeMaxTile];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = lane % LPH, sub = lane / LPH;
    const bool active = j * 8 < d;
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
            const __nv_bfloat16* src = hs.x + (t0 + t) * hs.stride;
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = item * run + u * HPW + sub;
                x[u] = make_uint4(0u, 0u, 0u, 0u);
                if (active && h < hs.n_heads) x[u] = *reinterpret_cast<const uint4*>(src + (int64_t)h * d + j * 8);
            }
            float A[8], B[8];
            if constexpr (set < 2) {
                const float4* from = reinterpret_cast<const float4*>(coef + (t * 2 + set) * (LPH * 16) + j * 16);
                float4 a0 = make_float4(0.f, 0.f, 0.f, 0.f), a1 = a0, b0 = a0, b1 = a0;
                if (active) { a0 = from[0]; a1 = from[1]; b0 = from[2]; b1 = from[3]; }
                A[0] = a0.x; A[1] = a0.y; A[2] = a0.z; A[3] = a0.w; A[4] = a1.x; A[5] = a1.y; A[6] = a1.z; A[7] = a1.w;
                B[0] = b0.x; B[1] = b0.y; B[2] = b0.z; B[3] = b0.w; B[4] = b1.x; B[5] = b1.y; B[6] = b1.z; B[7] = b1.w;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = item * run + u * HPW + sub;
                if (item * run + u * HPW >= hs.n_heads) break;  // (the same for the whole warp)
                float y[8];
                unpack8(x[u], y);
                if constexpr (set < 2) {
                    float r = 1.f;
                    if (hs.w != nullptr) {
                        float ss = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
                        r = rsqrtf(group_sum<LPH>(ss) / (float)d + eps);
                    }
                    float xp[8];
                    unpack8(rope_partner(x[u], partner, turned, rp.interleaved), xp);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = r * fmaf(y[e], A[e], xp[e] * B[e]);
                }
                if (!active || h >= hs.n_heads) continue;
                const int64_t at = (to_row * hs.n_heads + h) * d + j * 8;
                if constexpr (F8 && set > 0) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(to) + at) = pack8_e4m3(y);
                else *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(to) + at) = pack8(y);
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

// Gradients.  With g = (the transposed rotation of dy) and xh = x rstd:
//   dw = sum over tokens and heads of g xh,   dx = rstd (g w - xh mean(g w xh))      (w = none: dx = g)
// rstd is computed again from x: that is cheaper than keeping it.  A lane accumulates its eight elements of dw of
// both sets in registers over all its items; lanes and warps of a CTA join in a fixed order, CTAs leave a row each
// in the workspace and norm_rope_dw_kernel adds the rows in order, so equal calls give equal bits.
// Shared memory: [token][lane of the head][cos 0..7, signed sin 0..7].
struct RopeGrads {
    const __nv_bfloat16* dy;  // rows of n_heads*d, at dy + token*stride
    int64_t stride;
    __nv_bfloat16* dx;        // dense
};

template <int LPH>
__global__ void __launch_bounds__(kRopeThreads)
norm_rope_grad_kernel(RopeArgs rp, RopeHeads q, RopeHeads k, RopeGrads gq, RopeGrads gk, int64_t n_tokens, int d,
                      float eps, bool w32, const int64_t* __restrict__ positions, int tile, float* __restrict__ dw_rows) {
    constexpr int HPW = 32 / LPH, U = 2;
    extern __shared__ __align__(16) float coef[];  // [tile][LPH][16], then reused: [warps][2][LPH*8]
    __shared__ int64_t s_pos[kRopeMaxTile];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = lane % LPH, sub = lane / LPH;
    const bool active = j * 8 < d;
    const int half = rp.rot / 2;
    const bool turned = rp.freqs != nullptr && j * 8 < rp.rot;
    const int partner = sub * LPH + (j * 8 < half ? j + half / 8 : j - half / 8);
    const int run = U * HPW;
    const int n_q = (q.n_heads + run - 1) / run, n_k = (k.n_heads + run - 1) / run, n_all = n_q + n_k;
    const int first_plain = rp.freqs != nullptr ? rp.rot : 0;
    float w[2][8], dw[2][8];
#pragma unroll
    for (int set = 0; set < 2; ++set)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const void* from = set == 0 ? q.w : k.w;
            w[set][e] = active && from != nullptr ? weight_at(from, j * 8 + e, w32) : 1.f;
            dw[set][e] = 0.f;
        }
    for (int64_t t0 = (int64_t)blockIdx.x * tile; t0 < n_tokens; t0 += (int64_t)gridDim.x * tile) {
        const int nt = (int)min((int64_t)tile, n_tokens - t0);
        if (threadIdx.x < nt) s_pos[threadIdx.x] = positions != nullptr ? positions[t0 + threadIdx.x] : 0;
        __syncthreads();
        if (rp.freqs != nullptr)
            for (int e = threadIdx.x; e < nt * half; e += kRopeThreads) {
                const int t = e / half, i = e - t * half;
                float c, s;
                rope_angle(rp, s_pos[t], i, c, s);
                const int a = rope_first(rp, i), b = rope_second(rp, i);
                float* to = coef + t * (LPH * 16);
                to[(a >> 3) * 16 + (a & 7)] = c;
                to[(a >> 3) * 16 + 8 + (a & 7)] = s;
                to[(b >> 3) * 16 + (b & 7)] = c;
                to[(b >> 3) * 16 + 8 + (b & 7)] = -s;
            }
        for (int e = threadIdx.x; e < nt * (d - first_plain); e += kRopeThreads) {
            const int t = e / (d - first_plain), c = first_plain + e - t * (d - first_plain);
            float* to = coef + t * (LPH * 16) + (c >> 3) * 16 + (c & 7);
            to[0] = 1.f;
            to[8] = 0.f;
        }
        __syncthreads();
        auto heads = [&](const RopeHeads& hs, const RopeGrads& gs, const float (&w)[8], float (&dw)[8], int t, int item) {
            const bool norm = hs.w != nullptr;
            uint4 xv[U], gv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = item * run + u * HPW + sub;
                xv[u] = gv[u] = make_uint4(0u, 0u, 0u, 0u);
                if (active && h < hs.n_heads) {
                    gv[u] = *reinterpret_cast<const uint4*>(gs.dy + (t0 + t) * gs.stride + (int64_t)h * d + j * 8);
                    if (norm) xv[u] = *reinterpret_cast<const uint4*>(hs.x + (t0 + t) * hs.stride + (int64_t)h * d + j * 8);
                }
            }
            float c[8], s[8];
            {
                const float4* from = reinterpret_cast<const float4*>(coef + t * (LPH * 16) + j * 16);
                float4 c0 = make_float4(0.f, 0.f, 0.f, 0.f), c1 = c0, s0 = c0, s1 = c0;
                if (active) { c0 = from[0]; c1 = from[1]; s0 = from[2]; s1 = from[3]; }
                c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
                s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (item * run + u * HPW >= hs.n_heads) break;  // (the same for the whole warp)
                const int h = item * run + u * HPW + sub;
                float g[8], gp[8];
                unpack8(gv[u], g);
                unpack8(rope_partner(gv[u], partner, turned, rp.interleaved), gp);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = fmaf(g[e], c[e], gp[e] * s[e]);
                if (norm) {
                    float x[8], ss = 0.f, dot = 0.f;
                    unpack8(xv[u], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        ss = fmaf(x[e], x[e], ss);
                        dot = fmaf(g[e] * w[e], x[e], dot);
                    }
                    ss = group_sum<LPH>(ss);
                    dot = group_sum<LPH>(dot);
                    const float r = rsqrtf(ss / (float)d + eps);
                    const float m = dot / (float)d * r * r;  // times x = xh mean(g w xh)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (h < hs.n_heads) dw[e] = fmaf(g[e], x[e] * r, dw[e]);  // (eps = 0: r of an absent head is infinite)
                        g[e] = r * (g[e] * w[e] - x[e] * m);
                    }
                }
                if (active && h < hs.n_heads)
                    *reinterpret_cast<uint4*>(gs.dx + ((t0 + t) * hs.n_heads + h) * d + j * 8) = pack8(g);
            }
        };
        for (int it = warp; it < nt * n_all; it += kRopeWarps) {
            const int t = it / n_all;
            const int item = it - t * n_all;
            if (item < n_q) heads(q, gq, w[0], dw[0], t, item);
            else heads(k, gk, w[1], dw[1], t, item - n_q);
        }
        __syncthreads();
    }
    if (dw_rows == nullptr) return;
#pragma unroll
    for (int set = 0; set < 2; ++set)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int o = 16; o >= LPH; o >>= 1) dw[set][e] += __shfl_xor_sync(0xffffffffu, dw[set][e], o);
            if (sub == 0) coef[(warp * 2 + set) * (LPH * 8) + j * 8 + e] = dw[set][e];
        }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * d; e += kRopeThreads) {
        const int set = e / d, c = e - set * d;
        float sum = 0.f;
        for (int i = 0; i < kRopeWarps; ++i) sum += coef[(i * 2 + set) * (LPH * 8) + c];
        dw_rows[(int64_t)blockIdx.x * 2 * d + e] = sum;
    }
}

// dw[e] = sum over the CTAs' rows, 32 columns per CTA: 32 x 32 threads, each row class in order, then a tree.
__global__ void __launch_bounds__(1024)
norm_rope_dw_kernel(const float* __restrict__ rows, int n_rows, int d, float* __restrict__ dwq, float* __restrict__ dwk) {
    __shared__ float s[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x >> 5;
    float sum = 0.f;
    if (c < 2 * d)
        for (int r = r0; r < n_rows; r += 32) sum += rows[(int64_t)r * 2 * d + c];
    s[r0][threadIdx.x & 31] = sum;
    __syncthreads();
    const float total = warp_sum(s[threadIdx.x & 31][r0]);  // warp r0 owns column r0 of the 32
    const int col = blockIdx.x * 32 + r0;
    if ((threadIdx.x & 31) == 0 && col < 2 * d) {
        if (col < d) { if (dwq != nullptr) dwq[col] = total; }
        else if (dwk != nullptr) dwk[col - d] = total;
    }
}

}  // namespace msa
