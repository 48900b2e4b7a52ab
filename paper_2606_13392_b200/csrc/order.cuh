// What the selections of largest values share (tokens that stay in a cache, the next token).
#pragma once

#include "common.cuh"

namespace msa {

// Order of floats as whole numbers: larger key, larger value; both zeros alike; NaN below everything.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    if (x != x) return 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Exclusive sum over the CTA's threads (a multiple of 32, at most 1024); total in *all.  s: 33 words of shared memory.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* s, uint32_t* all) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    uint32_t upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t below = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += below;
    }
    __syncthreads();  // (the words may still be read from the call before)
    if (lane == 31) s[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        uint32_t x = lane < warps ? s[lane] : 0u;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t below = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += below;
        }
        s[lane] = x;
    }
    __syncthreads();
    *all = s[warps - 1];
    return upto - v + (warp > 0 ? s[warp - 1] : 0u);
}

}  // namespace msa
