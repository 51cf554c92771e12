// Rounding one value to the E4M3 grid by Def. 1 (shared by the quantizers).
#pragma once

#include "common.cuh"

namespace srq {

// Bits of a quantizer's mode: stochastic rounding (else to nearest), E4M3 grid (else integers), stochastic
// rounding with 8 random bits per element (integer grid only).
constexpr int MODE_SR = 1, MODE_E4M3 = 2, MODE_SR8 = 4;

// E4M3 grid: Def. 1 with the step of the binade of t = x * (1/D): for 2^e <= |t| < 2^(e+1) (e >= -6;
// smaller |t| use e = -6, the subnormal spacing) the step is 2^(e-3) and u = t 2^(3-e) is rounded to
// an integer q in [-16, 16] in fixed point with 24 fractional bits, as on the integer grid (quantize.cu).  With E = e + 127 the biased
// exponent of t, the code is sign | ((E - 120) << 3) + |q| - 8: |q| = 16 carries into the exponent
// field (next binade), |q| < 8 only occurs for E = 121 and gives the subnormal codes, q = 0 gives +0.
// Returns the code in the low byte.
template <int MODE, bool NOTTED = false>
__device__ __forceinline__ uint32_t quantize_e4m3(float x, float inv, uint32_t word, uint32_t sh) {
    // sh = 3 - k for the E4Mk grid (k mantissa bits; 0 for E4M3 itself): the step of binade e is
    // 2^(e-k), q counts those steps, and q << sh is the same value in the E4M3 code's units of 2^(e-3)
    const float t = __fmul_rn(x, inv);
    const uint32_t E = max((__float_as_uint(t) >> 23) & 0xFFu, 121u);          // |t| <= 448: E <= 135
    const float s = __fmul_rn(t, __uint_as_float((281u - sh - E) << 23));       // t 2^(k-e) 2^24, exact
    uint32_t sum;
    if constexpr ((MODE & MODE_SR) != 0) {
        const int c = __float2int_ru(s);
        asm("mad.hi.u32 %0, %1, 16777216, %2;" : "=r"(sum) : "r"(NOTTED ? word : ~word), "r"((uint32_t)c));
    } else {
        sum = (uint32_t)__float2int_rd(s) + 0x00800000u;
    }
    const int q = (int)sum >> 24;
    return ((uint32_t)q & 0x80u) | ((E << 3) + ((uint32_t)abs(q) << sh) - 968u);
}

}  // namespace srq
