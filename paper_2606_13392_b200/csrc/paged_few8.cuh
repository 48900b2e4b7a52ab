// Attention over a paged fp8 cache for sequences of a few rows (decode): the line of units, the partials and the merge
// are those of paged_attn.cuh, a tile of query rows is at most 16.  Bound by HBM.
//
// Why not the tcgen05 kernel: its operands come from shared memory, so fp8 tiles have to be read, widened and written
// back (64 KB for 32 KB of cache), with 128-row products for 8 or 16 rows; it reached 45 % of the copy bandwidth on 32
// sequences of 4K - 32K tokens (171 us; this kernel 101 - 112 us, 70 - 77 %).  Here the fragments of warp-level products are
// widened in registers: a producer warp streams K and V tiles (16 KB each) through a ring of six, two CTAs per SM, four
// consumer warps own 32 keys of every tile: S = Q K^T, softmax, O^T += V^T P^T, all in registers; the four warps' results
// join at the end of an item.  Fragment orders as in attn_decode_kv8_kernel: the contraction index of Q K^T and the row index of O^T are
// permuted to the order in which 16-bit shared-memory matrix loads hand out fp8 bytes.
// K, V and P are fp16 in the products (E4M3 -> fp16 is exact), Q is fp16 with a power of two taken out of each row and
// put back into the scale, P is held 2^10 up (see paged_attn.cuh for both).
#pragma once

#include "paged_attn.cuh"
#include "warp_mma.cuh"

namespace msa {

constexpr int kFewStages = 6, kFewThreads = 160, kFewCtas = 2;  // CTAs per SM
constexpr int kFewRows = 16;
constexpr float kFewShift = 10.f;

template <int HG>
struct FewSmem {
    alignas(1024) uint8_t tile[kFewStages][kPagedKeys * 128];  // [key][128 fp8], 128-byte swizzle
    float join[2][HG * 8 * 128 + HG * 16];                     // two warps' O, maxima and sums on their way to another
    alignas(8) uint64_t full[kFewStages], empty[kFewStages];
    PagedPlan plan;
    int abort;
};

// Barrier of the four consumer warps; true if `mine` is in all.
__device__ __forceinline__ bool few_agree(bool mine) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, r;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred r, 1, 128, p;\n\t"
        "selp.u32 %0, 1, 0, r;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)mine)
        : "memory");
    return all != 0;
}

// HG: half-groups of eight rows (1 or 2).
template <int HG>
__global__ void __launch_bounds__(kFewThreads, kFewCtas)
paged_few8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedAttnArgs a,
                  const __nv_bfloat16* __restrict__ q, int box_keys, double inv_grid, int* status) {
    constexpr uint32_t TILE = kPagedKeys * 128;
    constexpr int NT = 4, KS = 2;  // a warp's 32 keys: score tiles of 8, second-product steps of 16
    extern __shared__ __align__(1024) uint8_t paged_smem[];
    FewSmem<HG>& sm = *reinterpret_cast<FewSmem<HG>*>(paged_smem);
    if ((smem_u32(paged_smem) & 1023) != 0) {  // swizzled tiles need it; the same for every thread
        if (threadIdx.x == 0) {
            report_async(status, kAsyncBadIndex, 0x7FF);
            a.ends[blockIdx.x * 2] = make_int4(0, 0, 0, 0);  // (nothing to merge)
        }
        return;
    }
    // paged_attn_tc_kernel comes behind for the longer sequences: it shares nothing with this one, so its CTAs may take SMs
    // that are done here.
    if (a.max_len < a.n_tokens) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort = &sm.abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kFewStages; ++s) { mbar_init(&sm.full[s], 1); mbar_init(&sm.empty[s], 4); }
        sm.abort = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }
    paged_stretch(a, sm.plan, (int64_t)1 << 40, inv_grid, status);
    __syncthreads();
    PagedWalk walk(sm.plan.place[0], sm.plan.place[1]);
    PagedItem it{};

    if (warp == 4) {
        // ---------------- producer: one box per page (or 128 keys of a larger one), a lane each; K then V of every tile
        const int boxes = kPagedKeys / box_keys, nowhere = a.c.n_pages * a.c.page_size;  // reads as zeros
        PagedEnds e{};
        uint32_t t = 0;
        bool ok = true;
        if (const long long late = g_debug_producer_delay; late > 0) spin_cycles(late);  // tests only
        auto place_of = [&](int b) {
            const uint32_t key = (uint32_t)b * kPagedKeys + lane * box_keys, size = a.c.page_size;  // (below 2^31 + 128)
            if (lane >= boxes || key >= (uint32_t)it.kv) return nowhere;
            const uint32_t slot = key / size;
            const int page = a.c.table[(int64_t)it.seq * a.c.max_pages + slot];
            if (page < 0 || page >= a.c.n_pages) {
                report_async(status, kAsyncBadIndex, 0x702);
                return nowhere;
            }
            return page * a.c.page_size + (int)(key - slot * size);
        };
        while (walk.next(a, it)) {
            if (e.first == 0) e.first = it.lo == 0 ? 3 : (it.hi < it.nb ? 1 : 2);
            e.open = it.lo == 0 && it.hi < it.nb;
            e.q_row = it.q_row; e.tokens = it.n0; e.head = it.head;
            int where = ok ? place_of(it.lo) : 0;
            for (int b = it.lo; ok && b < it.hi; ++b) {
                const int where_next = b + 1 < it.hi ? place_of(b + 1) : 0;
                for (int kv = 0; kv < 2; ++kv, ++t) {
                    const uint32_t st = t % kFewStages, use = t / kFewStages;
                    if (use > 0 && !mbar_wait(&sm.empty[st], (use - 1) & 1, abort)) {
                        if (lane == 0) report_async(status, kAsyncTimeout, 0x711);
                        ok = false;
                        break;
                    }
                    if (lane == 0) mbar_arrive_expect_tx(&sm.full[st], TILE);
                    __syncwarp();
                    if (lane < boxes)
                        tma_load_3d(sm.tile[st] + lane * box_keys * 128, kv == 0 ? &tm_k : &tm_v, 0, it.head, where, &sm.full[st]);
                }
                where = where_next;
            }
        }
        if (lane == 0) {
            a.ends[blockIdx.x * 2] = make_int4(e.first, e.open, e.q_row, e.tokens);
            a.ends[blockIdx.x * 2 + 1] = make_int4(e.head, 0, 0, 0);
        }
        if (*abort != 0) spin_cycles(200000);
        return;
    }

    // ---------------- consumers
    const int g = lane >> 2, t4 = lane & 3, H_q = a.c.H_kv * a.G;
    uint32_t t = 0;
    bool ok = true;
    while (ok && walk.next(a, it)) {
        // A fragments of Q: row hg*8 + g of the tile is (token, head of the group); this lane's first pair of step ks is
        // d = 16 ks + 4 t4, +1, its second d + 2, + 3.
        uint32_t qa[8][4];
        float scale[HG];
        int row_lim[HG];  // last visible position of the row, -1 for rows that are not there
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qa[ks][0] = qa[ks][1] = qa[ks][2] = qa[ks][3] = 0u;
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            const int r = hg * 8 + g, tok = r / a.G, head = r - tok * a.G;
            const bool here = tok < it.n0;
            row_lim[hg] = here ? it.pos + tok : -1;
            uint2 raw[8];
            uint32_t most = 0;
            const __nv_bfloat16* from = q + ((int64_t)(it.q_row + (here ? tok : 0)) * H_q + it.head * a.G + (here ? head : 0)) * 128 + 4 * t4;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                raw[ks] = here ? *reinterpret_cast<const uint2*>(from + ks * 16) : make_uint2(0u, 0u);
                most = max(max(most, raw[ks].x & 0x7FFF0000u), max(raw[ks].y & 0x7FFF0000u, max(raw[ks].x << 17 >> 1, raw[ks].y << 17 >> 1)));
            }
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // the largest element goes to [2^14, 2^15): beyond, for rows below 2^-98, as far as 2^112 takes it
            const int e = most == 0 ? 0 : max((int)(most >> 23) - 127 - 14, -112);
            const float f = __uint_as_float((uint32_t)(127 - e) << 23);
            scale[hg] = a.scale_log2e * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                const float2 u = bf16x2_to_float2(raw[ks].x), v = bf16x2_to_float2(raw[ks].y);
                qa[ks][hg] = pack2_f16(u.x * f, u.y * f);
                qa[ks][2 + hg] = pack2_f16(v.x * f, v.y * f);
            }
        }
        float m_run[HG], l_part[HG], acc[HG][8][4];
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            m_run[hg] = -INFINITY; l_part[hg] = 0.f;
#pragma unroll
            for (int mt = 0; mt < 8; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[hg][mt][i] = 0.f;
        }
        for (int b = it.lo; b < it.hi; ++b) {
            const int key0 = warp * 32;                          // this warp's keys in the tile
            const int64_t tile0 = (int64_t)b * kPagedKeys;
            // ---- S
            uint32_t st = t % kFewStages;
            if (!mbar_wait(&sm.full[st], (t / kFewStages) & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x721);
                ok = false;
                break;
            }
            uint32_t tb = smem_u32(sm.tile[st]);
            float c[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
                const int key = key0 + nt * 8 + (lane & 7);
#pragma unroll
                for (int q4 = 0; q4 < 2; ++q4) {  // four 16-byte chunks (64 d) per load
                    uint32_t r4[4];
                    ldmatrix_x4(r4, dec_kv8_addr(tb, key, q4 * 4 + (lane >> 3)));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // chunk 4 q4 + j: this lane holds its bytes 4 t4 .. 4 t4 + 3 of key g
                        const int ks = q4 * 4 + j;
                        uint32_t b0, b1;
                        e4m3x4_to_f16x2x2(r4[j], b0, b1);
                        mma_m16n8k16_f16(c[nt], qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], b0, b1);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[st]);
            ++t;
            // ---- softmax of every row over this warp's keys
            uint32_t pb[HG][KS][2];
#pragma unroll
            for (int hg = 0; hg < HG; ++hg) {
                const int lim = (int)max(min((int64_t)row_lim[hg] - tile0, (int64_t)kPagedKeys), (int64_t)-1);
                float mx = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int key = key0 + nt * 8 + 2 * t4;
                    c[nt][2 * hg] = key <= lim ? c[nt][2 * hg] * scale[hg] : -INFINITY;
                    c[nt][2 * hg + 1] = key + 1 <= lim ? c[nt][2 * hg + 1] * scale[hg] : -INFINITY;
                    mx = fmaxf(mx, fmaxf(c[nt][2 * hg], c[nt][2 * hg + 1]));
                }
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const float m_new = fmaxf(m_run[hg], mx);
                const float m_use = (m_new == -INFINITY ? 0.f : m_new) - kFewShift;  // (nothing visible so far)
                float psum = 0.f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float p0 = ex2_approx(c[nt][2 * hg] - m_use), p1 = ex2_approx(c[nt][2 * hg + 1] - m_use);
                    psum += p0 + p1;
                    pb[hg][nt >> 1][nt & 1] = pack2_f16(p0, p1);
                }
                if (__any_sync(0xffffffffu, m_new > m_run[hg])) {  // some row's maximum moved
                    const float corr = m_run[hg] == -INFINITY ? 0.f : ex2_approx(m_run[hg] - m_new);
                    l_part[hg] *= corr;
                    // O^T columns of this lane are rows 2 t4, 2 t4 + 1 of the half-group: fetch their factors
                    const float corr0 = __shfl_sync(0xffffffffu, corr, 8 * t4), corr1 = __shfl_sync(0xffffffffu, corr, 8 * t4 + 4);
#pragma unroll
                    for (int mt = 0; mt < 8; ++mt) {
                        acc[hg][mt][0] *= corr0; acc[hg][mt][1] *= corr1;
                        acc[hg][mt][2] *= corr0; acc[hg][mt][3] *= corr1;
                    }
                }
                l_part[hg] += psum;
                m_run[hg] = m_new;
            }
            // ---- O^T[d][row] += V^T[d][key] P^T[key][row]
            st = t % kFewStages;
            if (!mbar_wait(&sm.full[st], (t / kFewStages) & 1, abort)) {
                if (lane == 0) report_async(status, kAsyncTimeout, 0x722);
                ok = false;
                break;
            }
            tb = smem_u32(sm.tile[st]);
            const int v_lim = (int)min((int64_t)it.kv - 1 - tile0, (int64_t)kPagedKeys);  // keys behind it may hold anything
            // Output tile mt = the 16 d of chunk mt; row g of the tile is d = 16 mt + 2g, row g + 8 is d = 16 mt + 2g + 1: a
            // transposed 16-bit load hands this lane both d of a pair for two keys, byte permutes split them.
#pragma unroll
            for (int mp = 0; mp < 4; ++mp) {  // pairs of output tiles: chunks 2 mp, 2 mp + 1
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int i = lane >> 3;  // matrix: keys (i & 1) * 8 .., chunk 2 mp + (i >> 1)
                    const int key = key0 + ks * 16 + (i & 1) * 8 + (lane & 7);
                    uint32_t r4[4];
                    ldmatrix_x4_trans(r4, dec_kv8_addr(tb, key, mp * 2 + (i >> 1)));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t lo = r4[half * 2], hi = r4[half * 2 + 1];  // keys 2 t4, 2 t4 + 1 and 8 + those
                        if (v_lim < kPagedKeys - 1) {
                            const int k0 = key0 + ks * 16 + 2 * t4;
                            lo = keep_visible_pair(lo, k0, v_lim);
                            hi = keep_visible_pair(hi, k0 + 8, v_lim);
                        }
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16x2x2(__byte_perm(lo, 0u, 0x3120), a0, a1);
                        e4m3x4_to_f16x2x2(__byte_perm(hi, 0u, 0x3120), a2, a3);
#pragma unroll
                        for (int hg = 0; hg < HG; ++hg)
                            mma_m16n8k16_f16(acc[hg][mp * 2 + half], a0, a1, a2, a3, pb[hg][ks][0], pb[hg][ks][1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[st]);
            ++t;
        }
        // ---- the four warps join: 2, 3 into 0, 1, then 1 into 0
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            l_part[hg] += __shfl_xor_sync(0xffffffffu, l_part[hg], 1);
            l_part[hg] += __shfl_xor_sync(0xffffffffu, l_part[hg], 2);
        }
#pragma unroll 1
        for (int half = 2; half >= 1; half >>= 1) {
            float* at = sm.join[warp & (half - 1)];
            float* ml = at + HG * 8 * 128;
            if (warp >= half && warp < 2 * half) {
#pragma unroll
                for (int hg = 0; hg < HG; ++hg) {
#pragma unroll
                    for (int mt = 0; mt < 8; ++mt)  // (a lane's own order: the other warp's same lane reads it)
                        *reinterpret_cast<float4*>(at + ((hg * 8 + mt) * 32 + lane) * 4) =
                            make_float4(acc[hg][mt][0], acc[hg][mt][1], acc[hg][mt][2], acc[hg][mt][3]);
                    if (t4 == 0) { ml[hg * 16 + g] = m_run[hg]; ml[hg * 16 + 8 + g] = l_part[hg]; }
                }
            }
            ok = few_agree(ok);  // (a wait may run out in one warp and not in another: all go on or none)
            if (warp < half) {
#pragma unroll
                for (int hg = 0; hg < HG; ++hg) {
                    const float m_o = ml[hg * 16 + g], l_o = ml[hg * 16 + 8 + g], m_new = fmaxf(m_run[hg], m_o);
                    const float w0 = m_run[hg] == -INFINITY ? 0.f : ex2_approx(m_run[hg] - m_new);
                    const float w1 = m_o == -INFINITY ? 0.f : ex2_approx(m_o - m_new);
                    l_part[hg] = l_part[hg] * w0 + l_o * w1;
                    m_run[hg] = m_new;
                    const float a0 = __shfl_sync(0xffffffffu, w0, 8 * t4), a1 = __shfl_sync(0xffffffffu, w0, 8 * t4 + 4);
                    const float b0 = __shfl_sync(0xffffffffu, w1, 8 * t4), b1 = __shfl_sync(0xffffffffu, w1, 8 * t4 + 4);
#pragma unroll
                    for (int mt = 0; mt < 8; ++mt) {
                        const float4 o = *reinterpret_cast<const float4*>(at + ((hg * 8 + mt) * 32 + lane) * 4);
                        acc[hg][mt][0] = acc[hg][mt][0] * a0 + o.x * b0; acc[hg][mt][1] = acc[hg][mt][1] * a1 + o.y * b1;
                        acc[hg][mt][2] = acc[hg][mt][2] * a0 + o.z * b0; acc[hg][mt][3] = acc[hg][mt][3] * a1 + o.w * b1;
                    }
                }
            }
            few_agree(true);  // the buffer is free again
        }
        if (!ok) break;
        if (warp != 0) continue;
        // ---- rows out: directly, or as a partial of a cut tile
        const bool partial = it.partial();
        const int64_t slot = (int64_t)blockIdx.x * 2 + (it.lo > 0 ? 0 : 1);
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            // (this lane's O^T columns: rows 2 t4 and 2 t4 + 1 of the half-group)
            const float l0 = __shfl_sync(0xffffffffu, l_part[hg], 8 * t4), l1 = __shfl_sync(0xffffffffu, l_part[hg], 8 * t4 + 4);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = hg * 8 + 2 * t4 + u, tok = r / a.G, head = r - tok * a.G;
                if (tok >= it.n0) continue;
                const float l = u == 0 ? l0 : l1, inv = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing is zero)
                const int64_t out_row = ((int64_t)it.q_row + tok) * H_q + it.head * a.G + head;
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) {  // rows g and g + 8 of an output tile are d and d + 1
                    const int d0 = mt * 16 + 2 * g;
                    if (partial)
                        *reinterpret_cast<float2*>(a.part_o + (slot * a.slot_rows + r) * 128 + d0) = make_float2(acc[hg][mt][u], acc[hg][mt][2 + u]);
                    else
                        *reinterpret_cast<uint32_t*>(a.out + out_row * 128 + d0) = pack2(acc[hg][mt][u] * inv, acc[hg][mt][2 + u] * inv);
                }
            }
            const int r = hg * 8 + g, tok = r / a.G;
            if (t4 == 0 && tok < it.n0) {
                // the maximum as the merge takes it: what P was formed against
                const float m = m_run[hg] == -INFINITY ? -INFINITY : m_run[hg] - kFewShift, l = l_part[hg];
                if (partial) a.part_ml[slot * a.slot_rows + r] = make_float2(m, l);
                else if (a.lse != nullptr)
                    a.lse[((int64_t)it.q_row + tok) * H_q + it.head * a.G + (r - tok * a.G)] =
                        l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
        }
    }
}

}  // namespace msa
