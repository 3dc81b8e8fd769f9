// Whole weights of logits: w = floor(2^31 exp((l - max) / T) + 1/2).  Sums of them are exact in 64-bit integers, whatever their order.
#pragma once

#include <cstdint>

#include "rlcs_rows.cuh"

namespace rlcs_rows {

typedef unsigned long long u64;

// The logit as compared: NaN counts as -inf (never drawn), -0 as +0.
__device__ __forceinline__ float clean(float f) { return fmaxf(f, -INFINITY) + 0.f; }

__device__ __forceinline__ float scaled(float x, float m, float inv_t) { return x == m ? 0.f : (x - m) * inv_t; }

// floor(2^31 e + 1/2) for 0 <= e <= 1.  Below 2^-10, nearly every logit of a wide row, one multiply-add rounded down leaves the
// whole number in the upper bits of its fraction; above, the 24 bits of e are shifted by its exponent and the last place rounded.
__device__ __forceinline__ uint32_t weight_of(float e) {
    if (e < 0x1p-10f) return (__float_as_uint(__fmaf_rd(e, 0x1p31f, 4194304.5f)) & 0x7fffffu) >> 1;
    const uint32_t u = __float_as_uint(e);
    const int down = 127 - (int)(u >> 23);
    const uint32_t frac = (u << 8) | 0x80000000u;
    return down == 0 ? frac : ((frac >> (down - 1)) + 1) >> 1;
}

// A temperature that is not above 0 (NaN too) takes the most likely entry; 1 / T stays finite, so that 0 stays 0 in what it multiplies.
__device__ __forceinline__ float inverse_of(float t) { return t > 0.f ? fminf(1.f / t, 3.4028235e38f) : 1.f; }

__device__ __forceinline__ u64 target_of(float uniform, u64 kept) {
    const double u = (double)uniform;
    const u64 t = u > 0. ? (u64)(u * (double)kept) : 0;
    return t < kept ? t : kept - 1;
}

}  // namespace rlcs_rows
