// Device helpers of the block-scaled operators: step sizes of a block, conversions to and from E4M3,
// the gated activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "grid_e4m3.cuh"

namespace srq {

constexpr int QBLK = 128;                    // values per step size
constexpr float E4M3_MAX = 448.0f;

__device__ __forceinline__ uint32_t abs_word(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
// max(|m|, |a|, |b|) in one instruction; a NaN among them gives a NaN with a positive pattern, so that the pattern
// of a block's maximum still orders as an unsigned number and shows values that are not finite.
__device__ __forceinline__ float absmax3(float m, float a, float b) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void note(uint32_t* status, uint32_t code) { if (status) record_status(status, code); }

// Step size and reciprocal of a block from the bit pattern of its absmax m: the rule of the other quantizers with
// qmax = 448.  448 / m overflows binary32 exactly for m <= 7 * 2^-122, which stands for all zeros.
// The library's correctly rounded divisions took a good part of the kernels' time where a few threads divide and
// the rest wait.  In the range where nothing over- or underflows both quotients are formed from an approximation
// and the sign or size of the exact residual (a - q b in one fused multiply-add; Markstein, IBM J. Res. Dev.
// 34(1), 1990):
//   inv  = largest q with q m <= 448: after one correction q is at most one unit off, and the residuals of q and of
//          its upper neighbour say which of the three numbers it is;
//   step = m / 448 to nearest: q = m c, c = 1 / 448 to nearest, corrected once.
constexpr float DIV_LO = 0x1p-100f, DIV_HI = 0x1p100f;
__device__ __forceinline__ float block_inv(uint32_t amax_bits) {
    const float m = __uint_as_float(amax_bits);
    if (m > DIV_LO && m < DIV_HI) {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(m));
        float q = __fmul_rn(E4M3_MAX, r);
        q = __fmaf_rn(__fmaf_rn(-q, m, E4M3_MAX), r, q);
        const float up = __uint_as_float(__float_as_uint(q) + 1u), down = __uint_as_float(__float_as_uint(q) - 1u);
        return __fmaf_rn(-up, m, E4M3_MAX) >= 0.0f ? up : __fmaf_rn(-q, m, E4M3_MAX) >= 0.0f ? q : down;
    }
    return m > 0x1.Cp-120f ? __fdiv_rz(E4M3_MAX, m) : 0.0f;
}
__device__ __forceinline__ float block_size(uint32_t amax_bits) {
    const float m = __uint_as_float(amax_bits);
    if (m > DIV_LO && m < DIV_HI) {
        constexpr float c = 1.0f / 448.0f;
        const float q = __fmul_rn(m, c);
        return __fmaf_rn(__fmaf_rn(-E4M3_MAX, q, m), c, q);
    }
    return m > 0x1.Cp-120f ? __fdiv_rn(m, E4M3_MAX) : 0.0f;
}
__device__ __forceinline__ void block_step(uint32_t amax_bits, float* step, float* inv) {
    *inv = block_inv(amax_bits);
    *step = block_size(amax_bits);
}
// One NaN or infinite value makes the block's absmax (compared as an unsigned pattern) reach this.
__device__ __forceinline__ bool block_nonfinite(uint32_t amax_bits) { return amax_bits >= 0x7F800000u; }

// Four quotients to E4M3, nearest even, first in the low byte.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n.reg .b16 lo, hi;\n"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        "mov.b32 %0, {lo, hi};\n}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
// Four E4M3 codes to binary32 (exact, through binary16).
__device__ __forceinline__ void e4m3x4_to_f32(uint32_t w, float v[4]) {
    uint32_t lo, hi;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\n"
        "cvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}

// act(g) and act'(g) through the logistic function p = 1 / (1 + e^-z):
//   SiLU         z = g            act = g p     act' = p + g p (1 - p)
//   GELU (tanh)  z = 2 u(g)       act = g p     act' = p + g p (1 - p) 2 u'(g),   u = c (g + 0.044715 g^3)
// ((1 + tanh u) / 2 = 1 / (1 + e^-2u): no cancellation for negative g).  e^-z overflows to infinity for
// very negative z, and p is then 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// p of two values; dz: z'(g), GELU only (it is 1 for SiLU).
template <bool GELU>
__device__ __forceinline__ float2 logistic2(float2 g, float2* dz) {
    const float2 minus_log2e = make_float2(-1.4426950408889634f, -1.4426950408889634f), one = make_float2(1.0f, 1.0f);
    float2 z = g;
    if constexpr (GELU) {
        const float c = 1.5957691216057308f, k = 0.044715f;      // 2 sqrt(2 / pi)
        const float2 c2 = make_float2(c, c), gg = __fmul2_rn(g, g);
        z = __fmul2_rn(__fmul2_rn(c2, g), __ffma2_rn(make_float2(k, k), gg, one));
        // where g^2 is out of range g p (1 - p) is exactly 0: a finite slope keeps 0 times infinity out of the gradient.
        // (z' passes 1e30 from |g| = 2e15 on, and p is exactly 0 or 1 from |g| = 12 on.)
        const float2 d = __fmul2_rn(c2, __ffma2_rn(make_float2(3.0f * k, 3.0f * k), gg, one));
        *dz = make_float2(fminf(d.x, 1e30f), fminf(d.y, 1e30f));
    }
    const float2 e = __fmul2_rn(z, minus_log2e);
    const float2 d = __fadd2_rn(make_float2(exp2_fast(e.x), exp2_fast(e.y)), one);
    return make_float2(rcp_fast(d.x), rcp_fast(d.y));
}
// act(g) * u of two values.
template <bool GELU>
__device__ __forceinline__ float2 gated2(float2 g, float2 u) {
    float2 unused;
    return __fmul2_rn(__fmul2_rn(g, logistic2<GELU>(g, &unused)), u);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight consecutive elements of a row starting at column c; columns >= cols read as 0.  vec: base and pitch
// allow 16-byte loads of whole groups.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, bool vec, float v[8]) {
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + c);
            v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
            v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (c + e < cols) ? (float)row[c + e] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, bool vec, const float v[8]) {
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t*>(&p);
            }
            *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) row[c + e] = (T)v[e];
    }
}
// Eight codes of a row starting at column c (a multiple of 8; base and pitch are multiples of 16).
__device__ __forceinline__ void store_codes8(uint8_t* row, int64_t c, int64_t cols, uint32_t lo, uint32_t hi) {
    if (c + 8 <= cols) {
        *reinterpret_cast<uint2*>(row + c) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) row[c + e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
    }
}

// Thresholds (Philox words) of eight consecutive elements whose flat indices start at i0.
__device__ __forceinline__ void thresholds8(uint64_t i0, const PhiloxKeys& K, uint32_t rnd[8]) {
    if ((i0 & 3u) == 0) {
        const uint64_t j = i0 >> 2;
        philox_rounds((uint32_t)j, (uint32_t)(j >> 32), K, rnd);
        philox_rounds((uint32_t)(j + 1), (uint32_t)((j + 1) >> 32), K, rnd + 4);
    } else {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            uint32_t w[4];
            const uint64_t i = i0 + e, j = i >> 2;
            philox_rounds((uint32_t)j, (uint32_t)(j >> 32), K, w);
            const uint32_t sel = (uint32_t)i & 3u;
            const uint32_t word = sel == 0 ? w[0] : sel == 1 ? w[1] : sel == 2 ? w[2] : w[3];
#pragma unroll
            for (int s = 0; s < 8; ++s) if (s == e) rnd[s] = word;      // constant register indices
        }
    }
}
// Four values to codes with reciprocal step inv: SR with the given thresholds, else nearest even.
template <bool SR>
__device__ __forceinline__ uint32_t encode4(const float v0, const float v1, const float v2, const float v3,
                                            float i0, float i1, float i2, float i3, const uint32_t r0, const uint32_t r1,
                                            const uint32_t r2, const uint32_t r3) {
    if constexpr (SR) {
        const uint32_t c0 = quantize_e4m3<MODE_SR | MODE_E4M3>(v0, i0, r0, 0), c1 = quantize_e4m3<MODE_SR | MODE_E4M3>(v1, i1, r1, 0);
        const uint32_t c2 = quantize_e4m3<MODE_SR | MODE_E4M3>(v2, i2, r2, 0), c3 = quantize_e4m3<MODE_SR | MODE_E4M3>(v3, i3, r3, 0);
        return __byte_perm(__byte_perm(c0, c1, 0x0040), __byte_perm(c2, c3, 0x0040), 0x5410);
    } else {
        const float2 a = __fmul2_rn(make_float2(v0, v1), make_float2(i0, i1)), b = __fmul2_rn(make_float2(v2, v3), make_float2(i2, i3));
        return e4m3x4(a.x, a.y, b.x, b.y);
    }
}

}  // namespace srq
