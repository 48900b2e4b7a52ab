// Warp-level matrix plumbing shared by the streaming kernels of few query rows (decode, paged attention).
#pragma once

#include "common.cuh"

namespace msa {

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t smem_addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(smem_addr));
}

__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t smem_addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(smem_addr));
}

// A register of a transposed V fragment holds one d of two consecutive keys (`key` in the low
// half, `key + 1` in the high half).  Keys past `lim` are not part of the sequence: their P is
// exactly 0, but the cache rows there may be uninitialised (NaN or Inf), and 0 * NaN is NaN, so
// their V values are replaced with zeros.
__device__ __forceinline__ uint32_t keep_visible_pair(uint32_t v, int key, int lim) {
    return (key <= lim ? (v & 0x0000FFFFu) : 0u) | (key + 1 <= lim ? (v & 0xFFFF0000u) : 0u);
}

// 16-byte chunk `chunk` (0..7: d = 16 chunk .. 16 chunk + 15) of key row `key` inside a swizzled fp8 tile.
__device__ __forceinline__ uint32_t dec_kv8_addr(uint32_t tile_base, int key, int chunk) {
    return tile_base + (uint32_t)(key * 128 + ((chunk ^ (key & 7)) << 4));
}

__device__ __forceinline__ void mma_m16n8k16_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                  uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_m16n8k16_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

}  // namespace msa
