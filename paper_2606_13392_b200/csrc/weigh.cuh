// The attention weight that cached tokens receive (include/msa.h: msa_paged_weights): for every place j of a sequence and
// every KV head,
//   w[j] = (j was there before ? decay w[j] : 0) + sum over new tokens i that see j, query heads h of the group
//                                                  exp(scale <q[i, h], k_j> - lse[i, h])
// i.e. the column sums of the softmax whose row statistics the attention call has returned: no maximum to keep, one pass
// over the keys.
#pragma once

#include "norm_rope.cuh"
#include "tc_common.cuh"
#include "warp_mma.cuh"

namespace msa {

struct WeighArgs {
    PagedView c;
    const void* k;
    const __nv_bfloat16* q;  // [n_tokens, H_kv*G, d]
    const float* lse;        // [n_tokens, H_kv*G]
    float* w;                // [n_pages, H_kv, page_size]
    int G, n_tokens;
    int min_len, max_len;    // new tokens of the sequences that this launch takes
    float scale_log2e, decay;
};

// Places of a sequence, as far as 32-bit numbers go with a tile or two to spare.
__host__ __device__ __forceinline__ int64_t paged_places(const PagedView& c) {
    const int64_t n = (int64_t)c.max_pages * c.page_size, most = 2147483648ll - 65536;
    return n < most ? n : most;
}

struct WeighSeq { int q_row, q_len, kv, base; };  // base: position of the first new token; earlier places were there before

__device__ __forceinline__ WeighSeq weigh_seq(const WeighArgs& a, int s) {
    WeighSeq q;
    const int lo = max(a.c.cu_q[s], 0), end = a.c.cu_q[s + 1], hi = min(end, a.n_tokens);  // (rows that are not there: none)
    q.q_row = lo;
    q.q_len = max(hi - lo, 0);
    if (q.q_len < a.min_len || q.q_len > a.max_len) q.q_len = 0;  // (another launch's)
    q.kv = (int)min((int64_t)max(a.c.kv_lens[s], 0), paged_places(a.c));
    q.base = q.kv - max(end - lo, 0);
    return q;
}

// Where a place is: row of the key pool (page * page_size + slot; -1: nowhere) and index of its weight.
struct WeighPlace { int64_t row, w; };
__device__ __forceinline__ WeighPlace weigh_place(const WeighArgs& a, int s, int head, int key, int* status) {
    const uint32_t size = a.c.page_size, slot = (uint32_t)key / size;
    const int page = a.c.table[(int64_t)s * a.c.max_pages + slot];
    if (page < 0 || page >= a.c.n_pages) {
        report_async(status, kAsyncBadIndex, 0x802);
        return WeighPlace{-1, 0};
    }
    const int off = (int)((uint32_t)key - slot * size);
    return WeighPlace{(int64_t)page * size + off, ((int64_t)page * a.c.H_kv + head) * size + off};
}

__device__ __forceinline__ float weigh_old(const WeighArgs& a, int64_t at, int key, int base) {
    return a.decay != 0.f && key < base ? a.decay * a.w[at] : 0.f;
}

// ---------------------------------------------------------------- few rows
// Sequences of few new tokens (decode): bound by HBM, each key is read once.  A warp takes tiles of 16 keys: their 16 x 128
// elements go from memory straight to the registers of a product's first operand (a lane reads 16 bytes at a time; which
// element of the contraction a register holds is free, as long as the query fragments hold the same), 8 NT rows of
// queries (token, head of the group) are its second.  A key's sum is then spread over four lanes.  The next tile's loads
// are in flight meanwhile.  All tiles of all (sequence, head) form one line, of which every CTA takes an equal stretch.
// Measured (64/8 heads): 64 sequences of one token on up to 32K 386 - 405 us, 94 - 99 % of the copy bandwidth; on up to 1000
// 20 us; one token on 2K 4.8 us (latency: the stretch, places, keys, sums, one after the other).
constexpr int kWeighFewRows = 32;
constexpr int kWeighKeys = 16, kWeighWarps = 8, kWeighSegCost = 8;  // tiles' worth of a (sequence, head)'s beginning

struct WeighSpot { int seq, head, tile; };

struct WeighPlan {
    int64_t scan[kWeighWarps];
    WeighSpot spot[2];
};

__device__ __forceinline__ int weigh_tiles(const WeighSeq& q) { return q.q_len == 0 ? 0 : (q.kv + kWeighKeys - 1) / kWeighKeys; }

// This CTA's stretch: first place and end.  All threads call it; the plan is there after the next __syncthreads.
__device__ inline void weigh_stretch(const WeighArgs& a, WeighPlan& p, double inv_grid, int* status) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x < 2) p.spot[threadIdx.x] = WeighSpot{a.c.batch, 0, 0};
    const int per = (a.c.batch + (int)blockDim.x - 1) / (int)blockDim.x;
    const int lo = min((int)threadIdx.x * per, a.c.batch), hi = min(lo + per, a.c.batch);
    int64_t mine = 0;
    for (int s = lo; s < hi; ++s) {
        const int tiles = weigh_tiles(weigh_seq(a, s));
        if (tiles > 0) mine += (int64_t)a.c.H_kv * (tiles + kWeighSegCost);
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
    for (int w = 0; w < kWeighWarps; ++w) {
        if (w < warp) upto += p.scan[w];
        total += p.scan[w];
    }
    for (int e = 0; e < 2; ++e) {
        // (the same rounding in every CTA, not decreasing; the last one is the end whatever it says)
        int64_t u = (int64_t)((double)total * (double)(blockIdx.x + e) * inv_grid);
        if (blockIdx.x + e >= gridDim.x || u < upto - mine || u >= upto) continue;  // (one thread)
        u -= upto - mine;
        for (int s = lo; s < hi; ++s) {
            const int tiles = weigh_tiles(weigh_seq(a, s));
            const int64_t one = tiles + kWeighSegCost, all = tiles > 0 ? a.c.H_kv * one : 0;
            if (u < all) {
                const int head = (int)(u / one);
                p.spot[e] = WeighSpot{s, head, (int)min(u - head * one, (int64_t)tiles)};
                break;
            }
            u -= all;
        }
    }
}

__device__ __forceinline__ uint32_t weigh_f16x2(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// fp8 keys are half the bytes a tile: five tiles of a warp are on their way through shared memory instead, each lane's 16-byte
// pieces to places of its own, so that nothing is exchanged (32 sequences of 4K - 32K tokens, 64/4 heads: 135 us with one tile ahead in registers, 76 us, 64 % of the copy bandwidth).
constexpr int kWeighStages = 5;
struct WeighSlot {
    uint4 k[4][32];
    int64_t w[32];
    float old[32];
};
constexpr size_t weigh_few_smem(bool f8) { return f8 ? sizeof(WeighSlot) * kWeighStages * kWeighWarps : 0; }

template <int NT, bool F8>
__global__ void __launch_bounds__(kWeighWarps * 32, NT <= 2 ? 2 : 1)
weigh_few_kernel(const WeighArgs a, double inv_grid, int* status) {
    constexpr int LD = F8 ? 2 : 4;   // 16-byte loads of a key by a lane
    __shared__ WeighPlan plan;
    weigh_stretch(a, plan, inv_grid, status);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3, H_q = a.c.H_kv * a.G;
    const WeighSpot end = plan.spot[1];
    for (WeighSpot at = plan.spot[0]; at.seq < a.c.batch;) {
        const WeighSeq sq = weigh_seq(a, at.seq);
        const int tiles = weigh_tiles(sq);
        const bool last = at.seq == end.seq && at.head == end.head;
        const int hi = last ? end.tile : tiles;
        const int seq = at.seq, head = at.head;
        int t = at.tile + warp;
        if (last) at.seq = a.c.batch;
        else {
            at.tile = 0;
            if (tiles == 0 || ++at.head >= a.c.H_kv) {
                at.head = 0;
                ++at.seq;
                if (at.seq > end.seq) at.seq = a.c.batch;
            }
        }
        if (t >= hi) continue;

        // ---- a tile's places (of key lane mod 16), its keys
        struct Place { int row, off; };  // row of the pool (the host has seen that they are below 2^31), place in its page
        auto places_of = [&](int tile) {
            const uint32_t key = tile * kWeighKeys + (lane & 15), size = a.c.page_size, slot = key / size;
            Place p{-1, (int)(key - slot * size)};
            if (tile < hi && key < (uint32_t)sq.kv) {
                const int page = a.c.table[(int64_t)seq * a.c.max_pages + slot];
                if (page >= 0 && page < a.c.n_pages) p.row = page * (int)size + p.off;
                else report_async(status, kAsyncBadIndex, 0x802);
            }
            return p;
        };
        struct Tile { uint4 k[2][LD]; int64_t w; float old; };
        auto fetch = [&](const Place& p, int tile, Tile& x) {
            const int r0 = __shfl_sync(0xffffffffu, p.row, g), r1 = __shfl_sync(0xffffffffu, p.row, 8 + g);
            const int off = __shfl_sync(0xffffffffu, p.off, (t4 & 1) * 8 + g);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = i == 0 ? r0 : r1;
                const uint4* from = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.k) + ((int64_t)row * a.c.H_kv + head) * (F8 ? 128 : 256)) + t4;
#pragma unroll
                for (int j = 0; j < LD; ++j) x.k[i][j] = row >= 0 ? __ldg(from + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
            }
            // lanes 0 and 1 of four look after the weights of keys g and g + 8
            const int key = tile * kWeighKeys + (t4 & 1) * 8 + g;
            const int mine = t4 == 0 ? r0 : r1;
            x.w = t4 < 2 && mine >= 0 ? (int64_t)(mine - off) * a.c.H_kv + (int64_t)head * a.c.page_size + off : -1;
            x.old = x.w >= 0 ? weigh_old(a, x.w, key, sq.base) : 0.f;
        };

        // ---- 8 NT rows of queries
        uint32_t qf[NT][8][2];
        float nl[NT][2], sc[NT][2];
        int lim[NT][2];  // last visible place of the row, -1 for rows that are not there or are to give nothing
        auto load_q = [&](int first) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = first + n * 8 + g, tok = r / a.G, h = r - tok * a.G;
                const bool here = tok < sq.q_len;
                const uint4* from = reinterpret_cast<const uint4*>(a.q + ((int64_t)(sq.q_row + (here ? tok : 0)) * H_q + head * a.G + (here ? h : 0)) * 128);
                uint4 raw[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)  // the elements that the lane has of a key: 32 j + 8 t4 .., fp8: 64 (j / 2) + 16 t4 + 8 (j mod 2) ..
                    raw[j] = here ? __ldg(from + (F8 ? 8 * (j >> 1) + 2 * t4 + (j & 1) : 4 * j + t4)) : make_uint4(0u, 0u, 0u, 0u);
                float scale = a.scale_log2e;
                if constexpr (F8) {
                    // fp16 products: a power of two is taken out of a row so that its largest element is in [2^14, 2^15)
                    // (as far as 2^112 takes it), and put back into the scale
                    uint32_t most = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t v[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) most = max(most, max(v[i] & 0x7FFF0000u, v[i] << 17 >> 1));
                    }
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    const int e = most == 0 ? 0 : max((int)(most >> 23) - 127 - 14, -112);
                    const float f = __uint_as_float((uint32_t)(127 - e) << 23);
                    scale *= __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t v[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 u = bf16x2_to_float2(v[i]);
                            qf[n][2 * j + (i >> 1)][i & 1] = weigh_f16x2(u.x * f, u.y * f);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        qf[n][2 * j][0] = raw[j].x; qf[n][2 * j][1] = raw[j].y;
                        qf[n][2 * j + 1][0] = raw[j].z; qf[n][2 * j + 1][1] = raw[j].w;
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int rc = first + n * 8 + 2 * t4 + i, tc = rc / a.G, hc = rc - tc * a.G;
                    const bool there = tc < sq.q_len;
                    const float l = there ? __ldg(a.lse + (int64_t)(sq.q_row + tc) * H_q + head * a.G + hc) : INFINITY;
                    sc[n][i] = F8 ? __shfl_sync(0xffffffffu, scale, (2 * t4 + i) * 4) : scale;
                    nl[n][i] = -l * 1.4426950408889634f;
                    lim[n][i] = there && l != -INFINITY ? sq.base + tc : -1;  // (a row that saw nothing gives nothing, whatever it holds)
                }
            }
        };

        const int rows = sq.q_len * a.G;
        auto finish = [&](int tile, const Tile& x) {
            const int key0 = tile * kWeighKeys + g, key1 = key0 + 8;
            float s0 = 0.f, s1 = 0.f;
            // first operand: [16 of d][row g, row g + 8, and the same two elements on]
            uint32_t k[8][4];
#pragma unroll
            for (int j = 0; j < LD; ++j) {
                const uint32_t u[4] = {x.k[0][j].x, x.k[0][j].y, x.k[0][j].z, x.k[0][j].w};
                const uint32_t v[4] = {x.k[1][j].x, x.k[1][j].y, x.k[1][j].z, x.k[1][j].w};
                if constexpr (F8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e4m3x4_to_f16x2x2(u[i], k[4 * j + i][0], k[4 * j + i][2]);
                        e4m3x4_to_f16x2x2(v[i], k[4 * j + i][1], k[4 * j + i][3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        k[2 * j + i][0] = u[2 * i]; k[2 * j + i][1] = v[2 * i];
                        k[2 * j + i][2] = u[2 * i + 1]; k[2 * j + i][3] = v[2 * i + 1];
                    }
                }
            }
            for (int first = 0; first < rows; first += 8 * NT) {
                if (rows > 8 * NT) load_q(first);
                float part0 = 0.f, part1 = 0.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        if constexpr (F8) mma_m16n8k16_f16(c, k[ks][0], k[ks][1], k[ks][2], k[ks][3], qf[n][ks][0], qf[n][ks][1]);
                        else mma_m16n8k16_bf16(c, k[ks][0], k[ks][1], k[ks][2], k[ks][3], qf[n][ks][0], qf[n][ks][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float p0 = ex2_approx(fmaf(c[i], sc[n][i], nl[n][i])), p1 = ex2_approx(fmaf(c[2 + i], sc[n][i], nl[n][i]));
                        if (key0 <= lim[n][i]) part0 += p0;
                        if (key1 <= lim[n][i]) part1 += p1;
                    }
                }
                s0 += part0;
                s1 += part1;
            }
            s0 += __shfl_xor_sync(0xffffffffu, s0, 1);
            s1 += __shfl_xor_sync(0xffffffffu, s1, 1);
            s0 += __shfl_xor_sync(0xffffffffu, s0, 2);
            s1 += __shfl_xor_sync(0xffffffffu, s1, 2);
            if (x.w >= 0) a.w[x.w] = x.old + (t4 == 0 ? s0 : s1);
        };

        Place p = places_of(t);
        if constexpr (F8) {
            extern __shared__ __align__(16) uint8_t weigh_few_raw[];
            WeighSlot* slots = reinterpret_cast<WeighSlot*>(weigh_few_raw) + warp * kWeighStages;
            auto send = [&](int tile, int stage) {
                WeighSlot& x = slots[stage];
                const int r0 = __shfl_sync(0xffffffffu, p.row, g), r1 = __shfl_sync(0xffffffffu, p.row, 8 + g);
                const int off = __shfl_sync(0xffffffffu, p.off, (t4 & 1) * 8 + g);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = i == 0 ? r0 : r1;
                    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.k) + ((int64_t)max(row, 0) * a.c.H_kv + head) * 128) + t4;
#pragma unroll
                    for (int j = 0; j < LD; ++j)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(&x.k[i * LD + j][lane])), "l"(from + 4 * j), "r"(row >= 0 ? 16 : 0)
                                     : "memory");
                }
                const int key = tile * kWeighKeys + (t4 & 1) * 8 + g, mine = t4 == 0 ? r0 : r1;
                const int64_t w = t4 < 2 && mine >= 0 ? (int64_t)(mine - off) * a.c.H_kv + (int64_t)head * a.c.page_size + off : -1;
                const bool was = w >= 0 && a.decay != 0.f && key < sq.base;
                x.w[lane] = w;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(&x.old[lane])), "l"(a.w + (was ? w : 0)), "r"(was ? 4 : 0) : "memory");
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll
            for (int i = 0; i < kWeighStages - 1; ++i) {  // (tiles beyond the end: nowhere, nothing)
                send(t + i * kWeighWarps, i);
                p = places_of(t + (i + 1) * kWeighWarps);
            }
            if (rows <= 8 * NT) load_q(0);
            for (int stage = 0; t < hi; t += kWeighWarps) {
                const int ahead = stage == 0 ? kWeighStages - 1 : stage - 1;
                send(t + (kWeighStages - 1) * kWeighWarps, ahead);
                p = places_of(t + kWeighStages * kWeighWarps);
                asm volatile("cp.async.wait_group %0;" ::"n"(kWeighStages - 1) : "memory");
                Tile x;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < LD; ++j) x.k[i][j] = slots[stage].k[i * LD + j][lane];
                x.w = slots[stage].w[lane];
                x.old = a.decay * slots[stage].old[lane];
                finish(t, x);
                stage = stage + 1 == kWeighStages ? 0 : stage + 1;
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        } else {
            Tile x, y;
            fetch(p, t, x);
            p = places_of(t + kWeighWarps);
            if (rows <= 8 * NT) load_q(0);
            for (; t < hi; t += 2 * kWeighWarps) {  // two tiles in registers, taken in turn
                fetch(p, t + kWeighWarps, y);
                p = places_of(t + 2 * kWeighWarps);
                finish(t, x);
                if (t + kWeighWarps >= hi) break;
                fetch(p, t + 2 * kWeighWarps, x);
                p = places_of(t + 3 * kWeighWarps);
                finish(t + kWeighWarps, y);
            }
        }
    }
}

// ---------------------------------------------------------------- other head sizes
// A thread per key, the queries one after the other through shared memory; fp32 throughout.
template <bool F8>
__global__ void __launch_bounds__(128)
weigh_generic_kernel(const WeighArgs a, int d, int* status) {
    __shared__ float qs[256];
    const int H_q = a.c.H_kv * a.G;
    for (int64_t sh = blockIdx.y; sh < (int64_t)a.c.batch * a.c.H_kv; sh += gridDim.y) {
        const int s = (int)(sh / a.c.H_kv), head = (int)(sh - (int64_t)s * a.c.H_kv);
        const WeighSeq sq = weigh_seq(a, s);
        if (blockIdx.x == 0 && threadIdx.x == 0 && (a.c.kv_lens[s] < 0 || a.c.kv_lens[s] > paged_places(a.c)))
            report_async(status, kAsyncBadIndex, 0x801);
        if (sq.q_len == 0) continue;
        for (int64_t first = (int64_t)blockIdx.x * 128; first < sq.kv; first += (int64_t)gridDim.x * 128) {
            const int64_t key = first + threadIdx.x;
            const WeighPlace p = key < sq.kv ? weigh_place(a, s, head, (int)key, status) : WeighPlace{-1, 0};
            const uint8_t* row = static_cast<const uint8_t*>(a.k) + (p.row * a.c.H_kv + head) * d * (F8 ? 1 : 2);
            float sum = 0.f;
            for (int tok = (int)max((int64_t)0, first - sq.base); tok < sq.q_len; ++tok) {
                for (int h = 0; h < a.G; ++h) {
                    const int64_t at = (int64_t)(sq.q_row + tok) * H_q + head * a.G + h;
                    __syncthreads();
                    for (int c = threadIdx.x; c < d; c += 128) qs[c] = __bfloat162float(a.q[at * d + c]);
                    __syncthreads();
                    const float l = a.lse[at];
                    if (p.row < 0 || key > (int64_t)sq.base + tok || l == -INFINITY) continue;  // (a row that saw nothing gives nothing)
                    float x = 0.f;
                    for (int c = 0; c < d; ++c) x = fmaf(qs[c], idx_elem<F8>(row, c), x);
                    sum += exp2f(fmaf(x, a.scale_log2e, -l * 1.4426950408889634f));
                }
            }
            if (p.row >= 0) a.w[p.w] = weigh_old(a, p.w, (int)key, sq.base) + sum;
        }
    }
}

}  // namespace msa
