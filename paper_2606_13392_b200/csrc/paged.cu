// C ABI of what stands around the sparse path (see include/msa.h): norms of queries and keys with the position
// rotation and their gradients, the paged K/V cache, attention of new tokens over it.  Argument validation,
// launch shapes and dispatch; the arithmetic is in the kernels included below.
#include <algorithm>
#include <cmath>

#include "norm_rope.cuh"
#include "paged_attn.cuh"
#include "paged_few8.cuh"
#include "tc_common.cuh"

namespace msa {

bool paged_set_wait(long long limit, long long late) {
    return cudaMemcpyToSymbol(g_wait_limit_cycles, &limit, sizeof(limit)) == cudaSuccess &&
           cudaMemcpyToSymbol(g_debug_producer_delay, &late, sizeof(late)) == cudaSuccess;
}

static bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

static int current_device() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) cuda_failed();
    return dev < 0 || dev >= 64 ? 0 : dev;
}

static int sm_count() {
    static int n[64] = {0};  // per device
    const int dev = current_device();
    if (n[dev] == 0 && cudaDeviceGetAttribute(&n[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cuda_failed();
        n[dev] = 148;
    }
    return n[dev];
}

// The status word of the current device; its address is looked up once per device.
static int* status_word() {
    static int* word[64] = {nullptr};
    const int dev = current_device();
    if (word[dev] == nullptr) word[dev] = async_status_ptr();
    return word[dev];
}

// ---------------------------------------------------------------------- norm and rotation
static msa_status_t resolve_rope(const msa_rope_t* rope, int d, RopeArgs& rp) {
    rp = RopeArgs{nullptr, 0, 0, 1.f};
    if (d <= 0) return MSA_ERR_INVALID_ARG;
    if (d % 8 != 0 || d > 256) return MSA_ERR_UNSUPPORTED;
    if (rope == nullptr) return MSA_OK;
    if (rope->rot_dim < 0 || rope->rot_dim > d || (rope->interleaved != 0 && rope->interleaved != 1)) return MSA_ERR_INVALID_ARG;
    if (!std::isfinite(rope->mscale)) return MSA_ERR_INVALID_ARG;
    if (rope->rot_dim == 0) return MSA_OK;
    if (rope->freqs == nullptr || !aligned_to(rope->freqs, 8)) return MSA_ERR_INVALID_ARG;
    if (rope->rot_dim % (rope->interleaved ? 8 : 16) != 0) return MSA_ERR_UNSUPPORTED;
    rp = RopeArgs{rope->freqs, rope->rot_dim, rope->interleaved, rope->mscale};
    return MSA_OK;
}

// Rows of n_heads*d bf16 every `stride` elements.
static bool rows_ok(const void* x, int64_t stride, int64_t n_heads, int d) {
    return x != nullptr && aligned_to(x, 16) && stride % 8 == 0 && stride >= n_heads * d;
}
static bool weight_ok(const void* w, bool w32) { return w == nullptr || aligned_to(w, w32 ? 4 : 2); }

constexpr int kMaxRopeHeads = 1024;

// Lanes reserved for a head.
static int lanes_per_head(int d) { return d <= 64 ? 8 : (d <= 128 ? 16 : 32); }

// Launch shape.  Many tokens: as many a CTA at a time as make about nine items a warp (eight of 64 + 8 heads of 128), so
// that the angles' latency is paid once for them, within the shared memory of a launch.  Few: one a CTA, its items spread
// over CTAs until the machine has four CTAs per SM (each repeats the token's angles).  At most twice the CTAs that are
// resident: the second half evens out the rounds.
struct RopeGrid { int tile, per; dim3 grid; size_t smem; };
static RopeGrid rope_grid(int d, int H_q, int H_k, int H_v, int64_t n) {
    const int lanes = lanes_per_head(d), run = 4 * (32 / lanes);
    const int items = (H_q + run - 1) / run + (H_k + run - 1) / run + (H_v + run - 1) / run;
    const int64_t want = 4LL * sm_count();
    RopeGrid g;
    g.tile = rope_tile_limit(lanes);
    while (g.tile > 1 && (g.tile * items > 9 * kRopeWarps || ceil_div64(n, g.tile) < want * 3 / 4)) g.tile /= 2;
    const int64_t tiles = ceil_div64(n, g.tile);
    const int parts = tiles >= want ? 1 : (int)std::min<int64_t>(items, ceil_div64(want, tiles));
    g.per = (items + parts - 1) / parts;
    g.grid = dim3((unsigned)std::min<int64_t>(tiles, 2 * want), (items + g.per - 1) / g.per);
    g.smem = (size_t)g.tile * rope_token_bytes(lanes);
    return g;
}

template <int LPH, bool EXACT, bool APPEND, bool F8>
static void launch_norm_rope(const RopeArgs& rp, const RopeHeads& q, const RopeHeads& k, const RopeHeads& v, int64_t n,
                             int d, float eps, bool w32, const int64_t* positions, const PagedView& cache, void* k_pool,
                             void* v_pool, cudaStream_t st) {
    const RopeGrid g = rope_grid(d, q.n_heads, k.n_heads, v.n_heads, n);
    StageScope sc(kStageNone, st);
    norm_rope_kernel<LPH, EXACT, APPEND, F8><<<g.grid, kRopeThreads, g.smem, st>>>(rp, q, k, v, n, d, eps, w32, positions, g.tile, g.per,
                                                                                 cache, k_pool, v_pool, APPEND ? status_word() : nullptr);
}

template <bool APPEND, bool F8>
static msa_status_t run_norm_rope(const RopeArgs& rp, const RopeHeads& q, const RopeHeads& k, const RopeHeads& v,
                                  int64_t n, int d, float eps, bool w32, const int64_t* positions,
                                  const PagedView& cache, void* k_pool, void* v_pool, cudaStream_t st) {
#define MSA_ROPE(LPH, EXACT) launch_norm_rope<LPH, EXACT, APPEND, F8>(rp, q, k, v, n, d, eps, w32, positions, cache, k_pool, v_pool, st)
    const int lanes = lanes_per_head(d);
    if (d == 64) MSA_ROPE(8, true);
    else if (d == 128) MSA_ROPE(16, true);
    else if (lanes == 8) MSA_ROPE(8, false);
    else if (lanes == 16) MSA_ROPE(16, false);
    else MSA_ROPE(32, false);
#undef MSA_ROPE
    return launch_status();
}

// CTAs of the gradient kernel, each leaving a row of weight gradients: all that are resident at once, shared out by
// heads (the angles, which both kinds compute, cost a warp about as much as four heads).
struct GradGrid { int64_t ctas, q_ctas; };
static GradGrid grad_grid(int H_q, int H_k) {
    GradGrid g;
    g.ctas = (int64_t)kGradCtas * sm_count();
    g.q_ctas = H_k == 0 ? g.ctas : (H_q == 0 ? 0 : std::min<int64_t>(g.ctas - 1, std::max<int64_t>(1, g.ctas * (H_q + 4) / (H_q + H_k + 8))));
    return g;
}

template <int LPH, bool EXACT>
static void launch_norm_rope_grad(const RopeArgs& rp, const RopeHeads& q, const RopeHeads& k, const RopeGrads& gq,
                                  const RopeGrads& gk, int64_t n, int d, float eps, bool w32, const int64_t* positions,
                                  const GradGrid& g, float* dw_rows, cudaStream_t st) {
    const size_t smem = std::max(grad_smem<LPH>(), (size_t)kGradWarps * LPH * 8 * sizeof(float));
    StageScope sc(kStageNone, st);
    norm_rope_grad_kernel<LPH, EXACT><<<(unsigned)g.ctas, kGradThreads, smem, st>>>(rp, q, k, gq, gk, n, d, eps, w32, positions,
                                                                                   (int)g.q_ctas, dw_rows);
}

// ---------------------------------------------------------------------- the paged cache
static msa_status_t resolve_cache(const msa_paged_cache_t* c, int64_t n_tokens, PagedView& v) {
    if (c == nullptr || n_tokens < 0 || n_tokens > 2147483647LL) return MSA_ERR_INVALID_ARG;
    if (c->batch < 0 || c->max_pages < 0 || c->n_pages < 0 || c->page_size <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0)
        return MSA_ERR_INVALID_ARG;
    if ((c->fp8 != 0 && c->fp8 != 1) || c->max_new < 0) return MSA_ERR_INVALID_ARG;
    if (c->head_dim % 8 != 0 || c->head_dim > 256 || c->n_kv_heads > kMaxRopeHeads) return MSA_ERR_UNSUPPORTED;
    v = PagedView{c->cu_q, c->kv_lens, c->page_table, c->batch, c->max_pages, c->n_pages, c->page_size, c->n_kv_heads};
    if (c->batch == 0 || n_tokens == 0) return MSA_OK;
    if (!c->cu_q || !c->kv_lens || !aligned_to(c->cu_q, 4) || !aligned_to(c->kv_lens, 4)) return MSA_ERR_INVALID_ARG;
    if (c->max_pages > 0 && (!c->page_table || !aligned_to(c->page_table, 4))) return MSA_ERR_INVALID_ARG;
    if (c->n_pages > 0 && (!c->k || !aligned_to(c->k, 16) || !aligned_to(c->v, 16))) return MSA_ERR_INVALID_ARG;
    return MSA_OK;
}

// ---------------------------------------------------------------------- attention over the cache
// Workspace: the CTAs' ends, then the partials; the same for the small kernel where a call may use it.
struct PagedWorkspace { size_t ends, ml, o, few_ends, few_ml, few_o, bytes; };
static PagedWorkspace paged_workspace(bool few) {
    const size_t n = sm_count(), rows = 2 * n * kPagedSlotRows, few_ctas = few ? kFewCtas * n : 0, few_rows = 2 * few_ctas * kFewRows;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at += (bytes + 255) / 256 * 256; return from; };
    PagedWorkspace w;
    w.ends = take(n * sizeof(PagedEnds));
    w.ml = take(rows * sizeof(float2));
    w.o = take(rows * 128 * sizeof(float));
    w.few_ends = take(few_ctas * sizeof(PagedEnds));
    w.few_ml = take(few_rows * sizeof(float2));
    w.few_o = take(few_rows * 128 * sizeof(float));
    w.bytes = at;
    return w;
}
static void paged_place_workspace(PagedAttnArgs& a, void* workspace, size_t ends, size_t ml, size_t o) {
    a.ends = (int4*)((char*)workspace + ends);
    a.part_ml = (float2*)((char*)workspace + ml);
    a.part_o = (float*)((char*)workspace + o);
}

static int common_divisor(int a, int b) { return b == 0 ? a : common_divisor(b, a % b); }

// Shapes of the tensor-core kernel: one 128-wide head row, a group that fits 128 rows, pages that are whole
// 1 KB operand atoms (8 keys), coordinates in 32 bits.
static bool paged_tc_ok(const msa_paged_cache_t& c, int G) {
    return c.head_dim == 128 && G <= 128 && c.page_size % 8 == 0 && c.n_pages > 0 &&
           (int64_t)c.n_pages * c.page_size < 2147483647LL - 128;
}

// A launch that may begin before the one in front of it has ended.
template <class... Params, class... Args>
static msa_status_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    StageScope sc(kStageNone, st);
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? MSA_OK : cuda_failed();
}

// Merges the tiles that the boundaries between the CTAs of a launch cut, or of two (b).  A cut tile has at most slot_rows rows:
// up to 64 at a time, as far as the call has rows.  (The kernel waits for the attention kernels before it reads.)
static msa_status_t launch_paged_combine(const PagedAttnArgs& a, int ctas, const PagedAttnArgs* b, int b_ctas, cudaStream_t st) {
    const int64_t most = std::min<int64_t>(std::max(a.slot_rows, b != nullptr ? b->slot_rows : 0), (int64_t)a.n_tokens * a.G);
    const PagedCuts c0{a.part_o, a.part_ml, a.ends, a.TPT, a.slot_rows, ctas};
    const PagedCuts c1 = b != nullptr ? PagedCuts{b->part_o, b->part_ml, b->ends, b->TPT, b->slot_rows, b_ctas} : PagedCuts{};
    const dim3 grid(c0.n_ctas + c1.n_ctas, (unsigned)std::min<int64_t>(64 / kMergeWarps, ceil_div64(most, kMergeWarps)));
    return launch_early(b != nullptr ? paged_combine_kernel<true> : paged_combine_kernel<false>, grid, kMergeThreads, 0, st, a, c0, c1);
}

// Which kernels a call on an fp8 cache takes.  The small kernel (paged_few8.cuh) is the faster one for sequences whose rows
// one of its tiles holds; of a longer one it would read the keys once for every tile (255 single tokens and a chunk of 257
// on 28K, 8 heads per group: 1470 us on it alone, 510 us with the chunk on the tcgen05 kernel).  The lengths are on the device and
// a captured call follows them; the host knows their sum and count, and the caller may say the longest.
//   tokens: of the small kernel's tile: the eight or sixteen rows that hold the longest sequence, or the average one; 0:
//           not even sixteen do, the tcgen05 kernel takes all.
//   alone:  no sequence is longer than the tile, if what the caller says holds or none is empty: the small kernel takes all
//           (right for any lengths, and slow where that is not so: 256 tokens on 28K beside 255 empty sequences 1904 us
//           against 240).  Else each kernel takes the sequences of its lengths; a second launch that finds none costs 2 to
//           8 us (32 sequences of two tokens on 4K - 32K 215 -> 222 us).
struct PagedFew { int tokens; bool alone; };
static PagedFew paged_few8(const PagedAttnArgs& a, const msa_paged_cache_t& c) {
    if (c.fp8 != 1 || a.G > kFewRows) return PagedFew{0, false};
    const int longest = c.max_new > 0 ? std::min(c.max_new, a.n_tokens) : a.n_tokens;
    for (const int rows : {8, kFewRows})
        if (longest <= rows / a.G) return PagedFew{rows / a.G, true};
    for (const int rows : {8, kFewRows})
        if (a.n_tokens <= (int64_t)c.batch * (rows / a.G))
            return PagedFew{rows / a.G, c.max_new == 0 && a.n_tokens - (c.batch - 1) <= rows / a.G};
    return PagedFew{0, false};
}

template <int HG>
static msa_status_t launch_paged_few8(const PagedAttnArgs& a, const msa_paged_cache_t& c, const void* q, int grid, cudaStream_t st) {
    CUtensorMap tm_k, tm_v;
    const uint64_t H = (uint64_t)a.c.H_kv, rows = (uint64_t)c.n_pages * c.page_size;
    const int box = common_divisor(c.page_size, kPagedKeys);
    const uint64_t kd[3] = {64, H, rows}, ks[2] = {128, H * 128};  // (128 bytes of a key as 64 two-byte elements)
    const uint32_t kb[3] = {64, 1, (uint32_t)box};
    int* status = status_word();
    if (!encode_tmap_bf16(&tm_k, c.k, 3, kd, ks, kb, true) || !encode_tmap_bf16(&tm_v, c.v, 3, kd, ks, kb, true) || status == nullptr)
        return cuda_failed();
    const size_t smem = sizeof(FewSmem<HG>);
    static_assert(sizeof(FewSmem<HG>) <= 113 * 1024, "two CTAs per SM");
    static bool attr_set[64] = {false};  // per device
    const int dev = current_device();
    if (!attr_set[dev]) {
        if (cudaFuncSetAttribute(paged_few8_kernel<HG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
            return cuda_failed();
        attr_set[dev] = true;
    }
    {
        StageScope sc(kStageNone, st);
        paged_few8_kernel<HG><<<grid, kFewThreads, smem, st>>>(tm_k, tm_v, a, (const __nv_bfloat16*)q, box, 1.0 / grid, status);
    }
    return launch_status();
}

template <bool F8>
static msa_status_t launch_paged_attn(const PagedAttnArgs& a, const msa_paged_cache_t& c, const void* q, int grid, bool early,
                                      cudaStream_t st) {
    CUtensorMap tm_q, tm_q1, tm_k, tm_v;
    const uint64_t H_q = (uint64_t)a.c.H_kv * a.G, H = (uint64_t)a.c.H_kv, rows = (uint64_t)c.n_pages * c.page_size;
    const int box = std::min(common_divisor(c.page_size, kPagedKeys), F8 ? 32 : kPagedKeys);  // keys of a copy
    const uint64_t qd[3] = {128, H_q, (uint64_t)a.n_tokens}, qs[2] = {256, H_q * 256};
    const uint32_t qb[3] = {64, (uint32_t)a.G, (uint32_t)a.TPT}, qb1[3] = {64, (uint32_t)a.G, 1};
    bool ok = encode_tmap_bf16(&tm_q, q, 3, qd, qs, qb) && encode_tmap_bf16(&tm_q1, q, 3, qd, qs, qb1);
    if constexpr (F8) {  // (128 bytes of a key as 64 two-byte elements: only bytes move)
        const uint64_t kd[3] = {64, H, rows}, ks[2] = {128, H * 128};
        const uint32_t kb[3] = {64, 1, (uint32_t)box};
        ok = ok && encode_tmap_bf16(&tm_k, c.k, 3, kd, ks, kb, true) && encode_tmap_bf16(&tm_v, c.v, 3, kd, ks, kb, true);
    } else {  // 64 of d, 8 keys, the two halves of d, head, groups of 8 keys: a box is a run of operand atoms
        const uint64_t kd[5] = {64, 8, 2, H, rows / 8}, ks[4] = {H * 256, 128, 256, H * 2048};
        const uint32_t kb[5] = {64, 8, 2, 1, (uint32_t)box / 8};
        ok = ok && encode_tmap_bf16(&tm_k, c.k, 5, kd, ks, kb) && encode_tmap_bf16(&tm_v, c.v, 5, kd, ks, kb);
    }
    int* status = status_word();
    if (!ok || status == nullptr) return cuda_failed();
    const size_t smem = sizeof(PagedSmem);
    static bool attr_set[64] = {false};  // per device
    const int dev = current_device();
    if (!attr_set[dev]) {
        if (cudaFuncSetAttribute(paged_attn_tc_kernel<F8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
            return cuda_failed();
        attr_set[dev] = true;
    }
    // K and V of one (sequence, head) beyond a third of L2: CTAs on different tiles of it should read in step
    const int64_t snap = (int64_t)40e6 / (F8 ? 256 : 512);
    if (early)  // (behind the small kernel, which it shares nothing with)
        return launch_early(paged_attn_tc_kernel<F8>, grid, paged_threads(F8), smem, st, tm_q, tm_q1, tm_k, tm_v, a, box, snap,
                            1.0 / grid, status);
    StageScope sc(kStageNone, st);
    paged_attn_tc_kernel<F8><<<grid, paged_threads(F8), smem, st>>>(tm_q, tm_q1, tm_k, tm_v, a, box, snap, 1.0 / grid, status);
    return launch_status();
}

}  // namespace msa

using namespace msa;

extern "C" {

msa_status_t msa_qk_norm_rope(const msa_rope_t* rope, const void* q, int64_t q_stride, int32_t n_q_heads,
                              const void* q_weight, const void* k, int64_t k_stride, int32_t n_k_heads,
                              const void* k_weight, int32_t head_dim, int32_t weight_fp32, float eps,
                              const int64_t* positions, int64_t n_tokens, void* q_out, void* k_out,
                              msa_stream_t stream) {
    RopeArgs rp;
    const msa_status_t s = resolve_rope(rope, head_dim, rp);
    if (s != MSA_OK) return s;
    if (n_tokens < 0 || n_q_heads < 0 || n_k_heads < 0 || !(eps >= 0.f) || !std::isfinite(eps)) return MSA_ERR_INVALID_ARG;
    if (weight_fp32 != 0 && weight_fp32 != 1) return MSA_ERR_INVALID_ARG;
    if (n_q_heads > kMaxRopeHeads || n_k_heads > kMaxRopeHeads) return MSA_ERR_UNSUPPORTED;
    if (n_tokens == 0 || n_q_heads + n_k_heads == 0) return MSA_OK;
    const bool w32 = weight_fp32 == 1;
    if (n_q_heads > 0 && (!rows_ok(q, q_stride, n_q_heads, head_dim) || !rows_ok(q_out, (int64_t)n_q_heads * head_dim, n_q_heads, head_dim)))
        return MSA_ERR_INVALID_ARG;
    if (n_k_heads > 0 && (!rows_ok(k, k_stride, n_k_heads, head_dim) || !rows_ok(k_out, (int64_t)n_k_heads * head_dim, n_k_heads, head_dim)))
        return MSA_ERR_INVALID_ARG;
    if (!weight_ok(q_weight, w32) || !weight_ok(k_weight, w32)) return MSA_ERR_INVALID_ARG;
    if (rp.rot > 0 && (positions == nullptr || !aligned_to(positions, 8))) return MSA_ERR_INVALID_ARG;
    const RopeHeads qh{(const __nv_bfloat16*)q, q_stride, n_q_heads, q_weight, (__nv_bfloat16*)q_out};
    const RopeHeads kh{(const __nv_bfloat16*)k, k_stride, n_k_heads, k_weight, (__nv_bfloat16*)k_out};
    return run_norm_rope<false, false>(rp, qh, kh, RopeHeads{}, n_tokens, head_dim, eps, w32, positions, PagedView{}, nullptr,
                                       nullptr, (cudaStream_t)stream);
}

msa_status_t msa_norm_rope_plan(int32_t head_dim, int32_t n_q_heads, int32_t n_k_heads, int32_t n_v_heads, int64_t n_tokens,
                                int32_t* tile_tokens, int32_t* ctas, int32_t* parts, int32_t* shared_bytes) {
    if (head_dim <= 0 || n_q_heads < 0 || n_k_heads < 0 || n_v_heads < 0 || n_tokens <= 0) return MSA_ERR_INVALID_ARG;
    if ((int64_t)n_q_heads + n_k_heads + n_v_heads == 0) return MSA_ERR_INVALID_ARG;
    if (head_dim % 8 != 0 || head_dim > 256 || n_q_heads > kMaxRopeHeads || n_k_heads > kMaxRopeHeads || n_v_heads > kMaxRopeHeads)
        return MSA_ERR_UNSUPPORTED;
    const RopeGrid g = rope_grid(head_dim, n_q_heads, n_k_heads, n_v_heads, n_tokens);
    if (tile_tokens) *tile_tokens = g.tile;
    if (ctas) *ctas = (int32_t)g.grid.x;
    if (parts) *parts = (int32_t)g.grid.y;
    if (shared_bytes) *shared_bytes = (int32_t)g.smem;
    return MSA_OK;
}

msa_status_t msa_qk_norm_rope_backward_workspace_bytes(int32_t head_dim, int64_t n_tokens, size_t* min_bytes) {
    if (head_dim <= 0 || n_tokens < 0 || min_bytes == nullptr) return MSA_ERR_INVALID_ARG;
    if (head_dim % 8 != 0 || head_dim > 256) return MSA_ERR_UNSUPPORTED;
    *min_bytes = (size_t)grad_grid(1, 1).ctas * head_dim * sizeof(float);
    return MSA_OK;
}

msa_status_t msa_qk_norm_rope_backward(const msa_rope_t* rope, const void* dq_out, int64_t dq_stride,
                                       const void* dk_out, int64_t dk_stride, const void* q, int64_t q_stride,
                                       int32_t n_q_heads, const void* q_weight, const void* k, int64_t k_stride,
                                       int32_t n_k_heads, const void* k_weight, int32_t head_dim,
                                       int32_t weight_fp32, float eps, const int64_t* positions, int64_t n_tokens,
                                       void* dq, void* dk, float* dq_weight, float* dk_weight, void* workspace,
                                       size_t workspace_bytes, msa_stream_t stream) {
    RopeArgs rp;
    const msa_status_t s = resolve_rope(rope, head_dim, rp);
    if (s != MSA_OK) return s;
    if (n_tokens < 0 || n_q_heads < 0 || n_k_heads < 0 || !(eps >= 0.f) || !std::isfinite(eps)) return MSA_ERR_INVALID_ARG;
    if (weight_fp32 != 0 && weight_fp32 != 1) return MSA_ERR_INVALID_ARG;
    if (n_q_heads > kMaxRopeHeads || n_k_heads > kMaxRopeHeads) return MSA_ERR_UNSUPPORTED;
    const bool w32 = weight_fp32 == 1;
    const bool some = n_tokens > 0;
    if (some && n_q_heads > 0 &&
        (!rows_ok(dq_out, dq_stride, n_q_heads, head_dim) || !rows_ok(dq, (int64_t)n_q_heads * head_dim, n_q_heads, head_dim) ||
         (q_weight && !rows_ok(q, q_stride, n_q_heads, head_dim))))
        return MSA_ERR_INVALID_ARG;
    if (some && n_k_heads > 0 &&
        (!rows_ok(dk_out, dk_stride, n_k_heads, head_dim) || !rows_ok(dk, (int64_t)n_k_heads * head_dim, n_k_heads, head_dim) ||
         (k_weight && !rows_ok(k, k_stride, n_k_heads, head_dim))))
        return MSA_ERR_INVALID_ARG;
    if (!weight_ok(q_weight, w32) || !weight_ok(k_weight, w32)) return MSA_ERR_INVALID_ARG;
    if (some && rp.rot > 0 && (positions == nullptr || !aligned_to(positions, 8))) return MSA_ERR_INVALID_ARG;
    float* dwq = q_weight != nullptr ? dq_weight : nullptr;
    float* dwk = k_weight != nullptr ? dk_weight : nullptr;
    if (!aligned_to(dwq, 4) || !aligned_to(dwk, 4)) return MSA_ERR_INVALID_ARG;
    const bool want = dwq != nullptr || dwk != nullptr;
    const GradGrid g = grad_grid(n_q_heads, n_k_heads);
    if (want && some) {
        if (workspace == nullptr || !aligned_to(workspace, 16)) return MSA_ERR_INVALID_ARG;
        if (workspace_bytes < (size_t)g.ctas * head_dim * sizeof(float)) return MSA_ERR_WORKSPACE;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (some && n_q_heads + n_k_heads > 0) {
        const RopeHeads qh{(const __nv_bfloat16*)q, q_stride, n_q_heads, q_weight, nullptr};
        const RopeHeads kh{(const __nv_bfloat16*)k, k_stride, n_k_heads, k_weight, nullptr};
        const RopeGrads gq{(const __nv_bfloat16*)dq_out, dq_stride, (__nv_bfloat16*)dq};
        const RopeGrads gk{(const __nv_bfloat16*)dk_out, dk_stride, (__nv_bfloat16*)dk};
        float* dw = want ? (float*)workspace : nullptr;
#define MSA_GRAD(LPH, EXACT) launch_norm_rope_grad<LPH, EXACT>(rp, qh, kh, gq, gk, n_tokens, head_dim, eps, w32, positions, g, dw, st)
        const int lanes = lanes_per_head(head_dim);
        if (head_dim == 64) MSA_GRAD(8, true);
        else if (head_dim == 128) MSA_GRAD(16, true);
        else if (lanes == 8) MSA_GRAD(8, false);
        else if (lanes == 16) MSA_GRAD(16, false);
        else MSA_GRAD(32, false);
#undef MSA_GRAD
    }
    if (want) {
        const bool any = some && n_q_heads + n_k_heads > 0;  // no rows: the gradients are zeros
        StageScope sc(kStageNone, st);
        norm_rope_dw_kernel<<<dim3((head_dim + 31) / 32, 2), 1024, 0, st>>>((const float*)workspace, any ? (int)g.q_ctas : 0,
                                                                            any ? (int)g.ctas : 0, head_dim, dwq, dwk);
    }
    return launch_status();
}

msa_status_t msa_paged_append(const msa_paged_cache_t* cache, const msa_rope_t* rope, const void* q, int64_t q_stride,
                              int32_t n_q_heads, const void* q_weight, const void* k, int64_t k_stride,
                              const void* k_weight, const void* v, int64_t v_stride, int32_t weight_fp32, float eps,
                              int64_t n_tokens, void* q_out, msa_stream_t stream) {
    PagedView view;
    msa_status_t s = resolve_cache(cache, n_tokens, view);
    if (s != MSA_OK) return s;
    const int d = cache->head_dim, H = cache->n_kv_heads;
    RopeArgs rp;
    if ((s = resolve_rope(rope, d, rp)) != MSA_OK) return s;
    if (n_q_heads < 0 || !(eps >= 0.f) || !std::isfinite(eps)) return MSA_ERR_INVALID_ARG;
    if (weight_fp32 != 0 && weight_fp32 != 1) return MSA_ERR_INVALID_ARG;
    if (n_q_heads > kMaxRopeHeads) return MSA_ERR_UNSUPPORTED;
    if (n_tokens == 0 || cache->batch == 0) return MSA_OK;
    const bool w32 = weight_fp32 == 1;
    if (n_q_heads > 0 && (!rows_ok(q, q_stride, n_q_heads, d) || !rows_ok(q_out, (int64_t)n_q_heads * d, n_q_heads, d)))
        return MSA_ERR_INVALID_ARG;
    if (!rows_ok(k, k_stride, H, d)) return MSA_ERR_INVALID_ARG;
    if ((v == nullptr) != (cache->v == nullptr)) return MSA_ERR_INVALID_ARG;
    if (v != nullptr && !rows_ok(v, v_stride, H, d)) return MSA_ERR_INVALID_ARG;
    if (!weight_ok(q_weight, w32) || !weight_ok(k_weight, w32)) return MSA_ERR_INVALID_ARG;
    if (status_word() == nullptr) return cuda_failed();
    const RopeHeads qh{(const __nv_bfloat16*)q, q_stride, n_q_heads, q_weight, (__nv_bfloat16*)q_out};
    const RopeHeads kh{(const __nv_bfloat16*)k, k_stride, H, k_weight, nullptr};
    const RopeHeads vh{(const __nv_bfloat16*)v, v_stride, v != nullptr ? H : 0, nullptr, nullptr};
    if (cache->fp8)
        return run_norm_rope<true, true>(rp, qh, kh, vh, n_tokens, d, eps, w32, nullptr, view, cache->k, cache->v, (cudaStream_t)stream);
    return run_norm_rope<true, false>(rp, qh, kh, vh, n_tokens, d, eps, w32, nullptr, view, cache->k, cache->v, (cudaStream_t)stream);
}

msa_status_t msa_paged_attn_workspace_bytes(const msa_paged_cache_t* cache, int32_t n_q_heads, size_t* min_bytes) {
    PagedView view;
    const msa_status_t s = resolve_cache(cache, 0, view);
    if (s != MSA_OK) return s;
    if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0 || min_bytes == nullptr) return MSA_ERR_INVALID_ARG;
    const int G = n_q_heads / cache->n_kv_heads;
    *min_bytes = paged_tc_ok(*cache, G) ? paged_workspace(cache->fp8 == 1 && G <= kFewRows).bytes : 0;
    return MSA_OK;
}

msa_status_t msa_paged_attn(const msa_paged_cache_t* cache, const void* q, int32_t n_q_heads, int64_t n_tokens,
                            float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                            msa_stream_t stream) {
    PagedView view;
    const msa_status_t s = resolve_cache(cache, n_tokens, view);
    if (s != MSA_OK) return s;
    const int d = cache->head_dim;
    if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return MSA_ERR_INVALID_ARG;
    if (!(softmax_scale >= 0.f) || !std::isfinite(softmax_scale)) return MSA_ERR_INVALID_ARG;
    if (n_q_heads > kMaxRopeHeads) return MSA_ERR_UNSUPPORTED;
    if (n_tokens == 0 || cache->batch == 0) return MSA_OK;
    if (!rows_ok(q, (int64_t)n_q_heads * d, n_q_heads, d) || !rows_ok(out, (int64_t)n_q_heads * d, n_q_heads, d)) return MSA_ERR_INVALID_ARG;
    if (!aligned_to(lse, 4) || (cache->n_pages > 0 && cache->v == nullptr)) return MSA_ERR_INVALID_ARG;
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d);
    PagedAttnArgs a{};
    a.c = view;
    a.G = n_q_heads / cache->n_kv_heads;
    a.n_tokens = (int)n_tokens;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.out = (__nv_bfloat16*)out;
    a.lse = lse;
    cudaStream_t st = (cudaStream_t)stream;
    if (paged_tc_ok(*cache, a.G)) {
        a.TPT = 128 / a.G;
        a.tile_tokens = 2 * a.TPT;
        a.slot_rows = kPagedSlotRows;
        a.max_len = 2147483647;
        const PagedFew few = paged_few8(a, *cache);
        const PagedWorkspace w = paged_workspace(cache->fp8 == 1 && a.G <= kFewRows);
        if (workspace == nullptr || !aligned_to(workspace, 256)) return MSA_ERR_INVALID_ARG;
        if (workspace_bytes < w.bytes) return MSA_ERR_WORKSPACE;
        paged_place_workspace(a, workspace, w.ends, w.ml, w.o);
        const int ctas = sm_count(), few_ctas = kFewCtas * ctas;
        PagedAttnArgs f = a;
        msa_status_t s = MSA_OK;
        if (few.tokens > 0) {
            f.TPT = f.tile_tokens = few.tokens;
            f.slot_rows = kFewRows;
            if (!few.alone) { f.max_len = few.tokens; a.min_len = few.tokens + 1; }
            paged_place_workspace(f, workspace, w.few_ends, w.few_ml, w.few_o);
            s = few.tokens * a.G <= 8 ? launch_paged_few8<1>(f, *cache, q, few_ctas, st) : launch_paged_few8<2>(f, *cache, q, few_ctas, st);
            if (s != MSA_OK) return s;
            if (few.alone) return launch_paged_combine(f, few_ctas, nullptr, 0, st);
        }
        s = cache->fp8 ? launch_paged_attn<true>(a, *cache, q, ctas, few.tokens > 0, st) : launch_paged_attn<false>(a, *cache, q, ctas, false, st);
        if (s != MSA_OK) return s;
        return few.tokens > 0 ? launch_paged_combine(f, few_ctas, &a, ctas, st) : launch_paged_combine(a, ctas, nullptr, 0, st);
    }
    const int64_t grid = ceil_div64(n_tokens * n_q_heads, 4);
    if (grid > 2147483647LL) return MSA_ERR_UNSUPPORTED;
    int* status = status_word();
    if (status == nullptr) return cuda_failed();
    {
        StageScope sc(kStageNone, st);
        if (cache->fp8) paged_attn_generic_kernel<true><<<(unsigned)grid, 128, 0, st>>>(a, (const __nv_bfloat16*)q, cache->k, cache->v, d, status);
        else paged_attn_generic_kernel<false><<<(unsigned)grid, 128, 0, st>>>(a, (const __nv_bfloat16*)q, cache->k, cache->v, d, status);
    }
    return launch_status();
}

}  // extern "C"
