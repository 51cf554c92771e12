// AdamW step over many tensors at once (the formula and the formats of the 8-bit moments are in srq.h).
//
// The list of tensors travels in the kernel's parameters, so that a call needs no table on the device and can be recorded as it
// is.  Everything is read once and written once.
//   32-bit states: a warp takes groups of 256 elements, a lane eight neighbouring ones.  Bound by HBM: 44 M elements, all binary32 (28 bytes
//   each), 186 us = 6.6 TB/s, the rate of a copy.
//   8-bit states: a warp takes groups of 512, a lane sixteen neighbouring ones, so that a block of 128 (the unit of a step size) is eight
//   lanes, whose new moments stay in registers between their absmax and their codes.  With bfloat16 weights and gradients 10 bytes
//   move per element, but 54 instructions are issued per 32 elements (10 of them Philox), and neither side is saturated: the arithmetic is on
//   pairs, thresholds and codes are put together byte-wise, and the next group's bytes arrive in shared memory while one is worked on
//   (without that 813 us).  352 M elements: 733 - 840 us on different machines, 4.3 - 4.9 TB/s (0.65 - 0.74 of a copy's rate)
//   and 0.69 of the issue slots.
#include "train.cuh"

namespace srq {

// 8-bit states: 96 registers, five CTAs of four warps per SM (256 threads at 80 registers spill, at 128 there are too few warps:
// 907 and 940 us against 843 for eight layers).
template <bool STATE8> constexpr int ADAM_THREADS = STATE8 ? 128 : 256;
template <bool STATE8> constexpr int ADAM_RUN = STATE8 ? 16 : 4;   // groups a warp takes in a row, where there are many
template <bool STATE8> constexpr int ADAM_GROUP = STATE8 ? 512 : 256;      // elements a warp takes at a time

struct AdamEntry {
    void* p; const void* g; void* m; void* v; float* m_step; float* v_step;
    int64_t n;
    int64_t first;                              // groups of the tensors before it
};
struct AdamScalars {
    float beta1, keep1, beta2, keep2;           // keep: 1 - beta
    float eps, lr, weight_decay;
    float inv_bias1, inv_root_bias2;            // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t); step_device: ln beta1, ln beta2
    const float* lr_device; const int64_t* step_device; const float* grad_scale;
    uint32_t* status;
    int64_t step;
    uint32_t id_lo, id_hi;                      // tensor_id + index of the first tensor
    uint32_t k0[10], k1[10];                    // Philox round keys
};
template <int CAP>
struct AdamParams {
    AdamScalars s;
    int32_t count, run;
    int64_t groups;
    AdamEntry e[CAP];
};

// Eight elements of type T from a 16-byte aligned address, as binary32.
template <typename T>
__device__ __forceinline__ void read8(const void* base, int64_t i, float2 v[4]) {
    if constexpr (sizeof(T) == 4) {
        const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + i);
        const float4 a = q[0], b = q[1];
        v[0] = make_float2(a.x, a.y); v[1] = make_float2(a.z, a.w); v[2] = make_float2(b.x, b.y); v[3] = make_float2(b.z, b.w);
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(base) + i);
        v[0] = make_float2(bf16_lo(a.x), bf16_hi(a.x)); v[1] = make_float2(bf16_lo(a.y), bf16_hi(a.y));
        v[2] = make_float2(bf16_lo(a.z), bf16_hi(a.z)); v[3] = make_float2(bf16_lo(a.w), bf16_hi(a.w));
    }
}
__device__ __forceinline__ void write8(void* base, int64_t i, const float2 v[4]) {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + i);
    q[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    q[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
template <typename T>
__device__ __forceinline__ float read1(const void* base, int64_t i) { return (float)reinterpret_cast<const T*>(base)[i]; }

__device__ __forceinline__ float sqrt_fast(float x) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Reciprocal step of a block of second moments, whose largest number is 496: block_inv (blocks.cuh) with another constant.
// 496 / m overflows for m <= 31 * 2^-124.
constexpr float E4M4_MAX = 496.0f, E4M4_DEAD = 0x1.Fp-120f;
__device__ __forceinline__ float e4m4_inv(float m) {
    if (m > DIV_LO && m < DIV_HI) {
        float q = __fmul_rn(E4M4_MAX, rcp_fast(m));
        q = __fmaf_rn(__fmaf_rn(-q, m, E4M4_MAX), rcp_fast(m), q);
        const float up = __uint_as_float(__float_as_uint(q) + 1u), down = __uint_as_float(__float_as_uint(q) - 1u);
        return __fmaf_rn(-up, m, E4M4_MAX) >= 0.0f ? up : __fmaf_rn(-q, m, E4M4_MAX) >= 0.0f ? q : down;
    }
    return m > E4M4_DEAD ? __fdiv_rz(E4M4_MAX, m) : 0.0f;
}
// Step size of a block of moments: absmax times the reciprocal of the grid's largest number, one product.
__device__ __forceinline__ float moment_step(float m, float inv, float top_reciprocal) { return inv > 0.0f ? __fmul_rn(m, top_reciprocal) : 0.0f; }

// What a thread derives from the scalars once.
struct AdamNow {
    float rate, decay, root, gscale;            // lr / bias1, 1 - lr wd, 1 / sqrt(bias2), factor on gradients
    uint32_t t;                                 // number of the step, for the thresholds
    uint32_t refused;                           // why nothing is done, or 0
};
__device__ __forceinline__ AdamNow adam_now(const AdamScalars& s) {
    AdamNow n;
    float ib1 = s.inv_bias1, ib2 = s.inv_root_bias2;
    n.t = (uint32_t)s.step;
    bool no_step = false;
    if (s.step_device) {
        const int64_t t = *s.step_device;
        n.t = (uint32_t)t;
        no_step = t < 1;
        // 1 - beta^t = -(e^(t ln beta) - 1): no cancellation for betas near 1
        ib1 = 1.0f / -expm1f((float)t * ib1);
        ib2 = 1.0f / sqrtf(-expm1f((float)t * ib2));
    }
    const float lr = s.lr_device ? *s.lr_device : s.lr;
    n.rate = lr * ib1;
    n.decay = 1.0f - lr * s.weight_decay;
    n.root = ib2;
    n.gscale = s.grad_scale ? *s.grad_scale : 1.0f;
    n.refused = block_nonfinite(abs_word(n.gscale)) || block_nonfinite(abs_word(lr)) ? SRQ_ERR_NONFINITE : 0u;
    if (no_step) n.refused = SRQ_ERR_INVALID_ARG;
    return n;
}

// Sum of two pairs of products, each rounded once.  The products are packed, the sums are not: the assembler contracts a packed
// product and a packed sum into one fused operation, though both name their rounding (seen: moments one unit off).
__device__ __forceinline__ float2 sum2(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }
// New moments of two elements.
__device__ __forceinline__ void adam_moments(const AdamScalars& s, float2 g, float2& m, float2& v) {
    m = sum2(__fmul2_rn(m, make_float2(s.beta1, s.beta1)), __fmul2_rn(g, make_float2(s.keep1, s.keep1)));
    v = sum2(__fmul2_rn(v, make_float2(s.beta2, s.beta2)), __fmul2_rn(__fmul2_rn(g, g), make_float2(s.keep2, s.keep2)));
}
__device__ __forceinline__ float2 adam_weight(const AdamScalars& s, const AdamNow& n, float2 p, float2 m, float2 v) {
    const float2 d = __ffma2_rn(make_float2(sqrt_fast(v.x), sqrt_fast(v.y)), make_float2(n.root, n.root), make_float2(s.eps, s.eps));
    const float2 u = __fmul2_rn(m, make_float2(rcp_fast(d.x), rcp_fast(d.y)));
    return __ffma2_rn(u, make_float2(-n.rate, -n.rate), __fmul2_rn(p, make_float2(n.decay, n.decay)));
}
// Two bfloat16 numbers by cutting off 16 bits after a threshold was added to them: the low halves of w0 (for x.x) and w1.  The
// conversion instruction does just that with the halves of its random operand (tests/test_gpu_bf16_cut.py holds it to the bits, over
// every finite pattern).
__device__ __forceinline__ uint32_t bf16_pair_sr(float2 x, uint32_t w0, uint32_t w1) {
    uint32_t r;
    asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(r) : "f"(x.y), "f"(x.x), "r"(__byte_perm(w0, w1, 0x5410)));
    return r;
}
__device__ __forceinline__ uint32_t bf16_pair(float2 x) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Philox words of the four elements of block j.
__device__ __forceinline__ void adam_words(const AdamScalars& s, uint64_t j, uint32_t c2, uint32_t c3, uint32_t w[4]) {
    uint32_t x0 = (uint32_t)j, x1 = (uint32_t)(j >> 32), x2 = c2, x3 = c3;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * x0, p1 = (uint64_t)0xCD9E8D57u * x2;
        x0 = (uint32_t)(p1 >> 32) ^ x1 ^ s.k0[r];
        x1 = (uint32_t)p1;
        x2 = (uint32_t)(p0 >> 32) ^ x3 ^ s.k1[r];
        x3 = (uint32_t)p0;
    }
    w[0] = x0; w[1] = x1; w[2] = x2; w[3] = x3;
}

// The tensor of group u: the last one that begins at or before it (empty tensors begin where the next one does).
template <int CAP>
__device__ __forceinline__ int adam_find(const AdamParams<CAP>& a, int64_t u) {
    int k = 0;
    for (int hi = a.count; hi - k > 1;) {
        const int mid = (k + hi) >> 1;
        if (a.e[mid].first <= u) k = mid; else hi = mid;
    }
    return k;
}

// What both kernels walk: CTAs take chunks of run * WARPS groups, warp w the groups w, w + WARPS, ... of a chunk.  All of it is the
// same for the lanes of a warp.
template <int WARPS, int CAP>
struct AdamCursor {
    const AdamParams<CAP>& a;
    int warp, r = 0, k = -1;
    int64_t chunk, size, end = 0;                              // end: groups before the tensor after tensor k
    __device__ __forceinline__ explicit AdamCursor(const AdamParams<CAP>& params) : a(params) {
        warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0);
        size = (int64_t)a.run * WARPS;
        chunk = blockIdx.x * size;
    }
    // The next group and its tensor; false: there is none.
    __device__ __forceinline__ bool next(int64_t& group, int& tensor) {
        for (; chunk < a.groups; chunk += gridDim.x * size, r = 0) {
            group = chunk + r * WARPS + warp;
            if (r == a.run || group >= a.groups) continue;
            ++r;
            if (k < 0 || group >= end) {
                k = adam_find(a, group);
                end = k + 1 < a.count ? a.e[k + 1].first : a.groups;
            }
            tensor = k;
            return true;
        }
        return false;
    }
};

// P, G: types of weights and gradients.  SR: bfloat16 weights are rounded stochastically.
template <typename P, typename G, bool SR, int CAP>
__global__ void __launch_bounds__(ADAM_THREADS<false>) adamw_kernel(const __grid_constant__ AdamParams<CAP> a) {
    pdl_enter();
    constexpr bool WORDS = SR && sizeof(P) == 2;
    const AdamScalars& s = a.s;
    const AdamNow now = adam_now(s);
    if (now.refused) {
        if (threadIdx.x == 0 && blockIdx.x == 0) note(s.status, now.refused);
        return;
    }
    AdamCursor<ADAM_THREADS<false> / 32, CAP> at(a);
    int64_t group;
    int k;
    while (at.next(group, k)) {
        const AdamEntry& e = a.e[k];
        const int64_t i = (group - e.first) * ADAM_GROUP<false> + (threadIdx.x & 31) * 8;
        const int64_t left = e.n - i;                          // elements of this lane: min(left, 8), none or less: none
        if (left <= 0) continue;
        float2 p[4], g[4], m[4], v[4];
        if (left >= 8) {
            read8<G>(e.g, i, g);
            read8<P>(e.p, i, p);
            read8<float>(e.m, i, m);
            read8<float>(e.v, i, v);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const bool in = q < left;
                const float gg = in ? read1<G>(e.g, i + q) : 0.0f, pp = in ? read1<P>(e.p, i + q) : 0.0f;
                const float mm = in ? read1<float>(e.m, i + q) : 0.0f, vv = in ? read1<float>(e.v, i + q) : 0.0f;
                if (q & 1) { p[q >> 1].y = pp; g[q >> 1].y = gg; m[q >> 1].y = mm; v[q >> 1].y = vv; }
                else { p[q >> 1].x = pp; g[q >> 1].x = gg; m[q >> 1].x = mm; v[q >> 1].x = vv; }
            }
        }
        uint32_t w[8];
        if constexpr (WORDS) {
            const uint64_t id = (((uint64_t)s.id_hi << 32) | s.id_lo) + (uint64_t)k + ((uint64_t)now.t << 32);
            adam_words(s, (uint64_t)i >> 2, (uint32_t)id, (uint32_t)(id >> 32), w);
            adam_words(s, ((uint64_t)i >> 2) + 1, (uint32_t)id, (uint32_t)(id >> 32), w + 4);
        }
        float mmax = 0.0f, vmax = 0.0f;
        uint32_t pb[8];                                        // weights: bits of binary32 numbers, or in the first four of bfloat16 pairs
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            g[q] = __fmul2_rn(g[q], make_float2(now.gscale, now.gscale));
            adam_moments(s, g[q], m[q], v[q]);
            mmax = absmax3(mmax, m[q].x, m[q].y);
            vmax = absmax3(vmax, v[q].x, v[q].y);
            const float2 x = adam_weight(s, now, p[q], m[q], v[q]);
            if constexpr (sizeof(P) == 2) {
                pb[q] = WORDS ? bf16_pair_sr(x, w[2 * q], w[2 * q + 1]) : bf16_pair(x);
            } else {
                pb[2 * q] = __float_as_uint(x.x); pb[2 * q + 1] = __float_as_uint(x.y);
            }
        }
        if (block_nonfinite(abs_word(mmax)) || block_nonfinite(abs_word(vmax))) note(s.status, SRQ_ERR_NONFINITE);
        if (left >= 8) {
            if constexpr (sizeof(P) == 2) {
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(e.p) + i) = make_uint4(pb[0], pb[1], pb[2], pb[3]);
            } else {
                uint4* o = reinterpret_cast<uint4*>(reinterpret_cast<float*>(e.p) + i);
                o[0] = make_uint4(pb[0], pb[1], pb[2], pb[3]);
                o[1] = make_uint4(pb[4], pb[5], pb[6], pb[7]);
            }
            write8(e.m, i, m);
            write8(e.v, i, v);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (q >= left) continue;
                if constexpr (sizeof(P) == 2) reinterpret_cast<uint16_t*>(e.p)[i + q] = (uint16_t)(pb[q >> 1] >> (16 * (q & 1)));
                else reinterpret_cast<uint32_t*>(e.p)[i + q] = pb[q];
                reinterpret_cast<float*>(e.m)[i + q] = q & 1 ? m[q >> 1].y : m[q >> 1].x;
                reinterpret_cast<float*>(e.v)[i + q] = q & 1 ? v[q >> 1].y : v[q >> 1].x;
            }
        }
    }
}

// Sixteen elements of type T as they lie in memory: 8 words (bfloat16) or 16 (binary32).  wide: 32-byte aligned.
template <typename T> struct Raw16 { uint32_t w[4 * sizeof(T)]; };
template <typename T>
__device__ __forceinline__ void write16(void* base, int64_t i, const Raw16<T>& r, bool wide) {
    char* p = reinterpret_cast<char*>(base) + i * (int64_t)sizeof(T);
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        if (wide) {
            Word8 x;
#pragma unroll
            for (int q = 0; q < 8; ++q) x.w[q] = r.w[8 * h + q];
            store32(p + 32 * h, x);
        } else {
            *reinterpret_cast<uint4*>(p + 32 * h) = make_uint4(r.w[8 * h], r.w[8 * h + 1], r.w[8 * h + 2], r.w[8 * h + 3]);
            *reinterpret_cast<uint4*>(p + 32 * h + 16) = make_uint4(r.w[8 * h + 4], r.w[8 * h + 5], r.w[8 * h + 6], r.w[8 * h + 7]);
        }
    }
}
// Pair q (elements 2 q and 2 q + 1).
template <typename T>
__device__ __forceinline__ float2 pair_of(const Raw16<T>& r, int q) {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(r.w[2 * q]), __uint_as_float(r.w[2 * q + 1]));
    else return make_float2(bf16_lo(r.w[q]), bf16_hi(r.w[q]));
}
// The first `left` of sixteen elements, one by one; the others are zero.
template <typename T>
__device__ __forceinline__ Raw16<T> read_some(const void* base, int64_t i, int64_t left) {
    Raw16<T> r;
#pragma unroll
    for (int q = 0; q < (int)(4 * sizeof(T)); ++q) r.w[q] = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        if (q >= left) continue;
        if constexpr (sizeof(T) == 4) r.w[q] = reinterpret_cast<const uint32_t*>(base)[i + q];
        else r.w[q >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(base)[i + q] << (16 * (q & 1));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void write_some(void* base, int64_t i, const Raw16<T>& r, int64_t left) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        if (q >= left) continue;
        if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(base)[i + q] = r.w[q];
        else reinterpret_cast<uint16_t*>(base)[i + q] = (uint16_t)(r.w[q >> 1] >> (16 * (q & 1)));
    }
}
__device__ __forceinline__ uint4 read_codes(const void* base, int64_t i, int64_t left) {
    const uint8_t* p = reinterpret_cast<const uint8_t*>(base) + i;
    if (left >= 16) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 16; ++q) if (q < left) w[q >> 2] |= (uint32_t)p[q] << (8 * (q & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void write_codes(void* base, int64_t i, const uint32_t w[4], int64_t left) {
    uint8_t* p = reinterpret_cast<uint8_t*>(base) + i;
    if (left >= 16) { *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]); return; }
#pragma unroll
    for (int q = 0; q < 16; ++q) if (q < left) p[q] = (uint8_t)(w[q >> 2] >> (8 * (q & 3)));
}

// Four codes of the second moment (E4M4 without a sign) as numbers times 2^-8: shifted into place they are binary16 numbers, the
// grid's subnormal ones included.
__device__ __forceinline__ void e4m4x4_to_f32(uint32_t w, float2 v[2]) {
    const uint32_t a = __byte_perm(w, 0, 0x4140) << 6, b = __byte_perm(w, 0, 0x4342) << 6;
    v[0] = __half22float2(*reinterpret_cast<const __half2*>(&a));
    v[1] = __half22float2(*reinterpret_cast<const __half2*>(&b));
}
// The top bytes of four words.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// Two codes' worth of a pair of moments: quotients x * inv, times 2^-120, where binary32's exponent field is the grid's, subnormal
// numbers included, as bits.
__device__ __forceinline__ uint2 code_bits(float2 x, float inv) {
    const float2 t = __fmul2_rn(__fmul2_rn(x, make_float2(inv, inv)), make_float2(0x1p-120f, 0x1p-120f));
    return make_uint2(__float_as_uint(t.x), __float_as_uint(t.y));
}

// What a lane has of a whole group on its way through shared memory, in pieces of 16 bytes: weights, gradients, codes.  Piece j of
// lane l lies at [j][l], so that neighbouring lanes' pieces are neighbours.  A lane reads only what it has copied itself.
template <typename P, typename G>
struct Staged {
    static constexpr int PP = sizeof(P), GP = sizeof(G), PIECES = PP + GP + 2;      // sixteen elements of n bytes: n pieces
    uint4 piece[PIECES][32];
};
__device__ __forceinline__ void copy16(uint4* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
template <typename P, typename G>
__device__ __forceinline__ void stage(Staged<P, G>& b, const AdamEntry& e, int64_t i, int lane) {
    typedef Staged<P, G> S;
    const char* p = reinterpret_cast<const char*>(e.p) + i * (int64_t)sizeof(P);
    const char* g = reinterpret_cast<const char*>(e.g) + i * (int64_t)sizeof(G);
#pragma unroll
    for (int j = 0; j < S::PP; ++j) copy16(&b.piece[j][lane], p + 16 * j);
#pragma unroll
    for (int j = 0; j < S::GP; ++j) copy16(&b.piece[S::PP + j][lane], g + 16 * j);
    copy16(&b.piece[S::PP + S::GP][lane], reinterpret_cast<const char*>(e.m) + i);
    copy16(&b.piece[S::PP + S::GP + 1][lane], reinterpret_cast<const char*>(e.v) + i);
}

// One group of 512 elements of tensor e, sixteen per lane, with the step sizes sm and sv.  FULL: all of them are there, and staged.
template <typename P, typename G, bool SR, bool FULL>
__device__ __forceinline__ void adam8_group(const AdamScalars& s, const AdamNow& now, const AdamEntry& e, int64_t i, uint64_t id, float sm, float sv,
                                            const Staged<P, G>* b) {
    typedef Staged<P, G> S;
    const int lane = threadIdx.x & 31;
    const int64_t left = FULL ? 16 : e.n - i;                  // elements of this lane: min(left, 16), none or less: none
    Raw16<P> p;
    Raw16<G> g;
    uint4 mc = make_uint4(0, 0, 0, 0), vc = make_uint4(0, 0, 0, 0);
    if constexpr (FULL) {
#pragma unroll
        for (int j = 0; j < S::GP; ++j) {
            const uint4 x = b->piece[S::PP + j][lane];
            g.w[4 * j] = x.x; g.w[4 * j + 1] = x.y; g.w[4 * j + 2] = x.z; g.w[4 * j + 3] = x.w;
        }
        mc = b->piece[S::PP + S::GP][lane];
        vc = b->piece[S::PP + S::GP + 1][lane];
    } else {
        g = read_some<G>(e.g, i, left);
        p = read_some<P>(e.p, i, left);
        if (left > 0) {
            mc = read_codes(e.m, i, left);
            vc = read_codes(e.v, i, left);
        }
    }
    sv *= 256.0f;                                              // with the decoder's 2^-8; at most 2^127
    float2 m[8], v[8];
    const uint32_t mw[4] = {mc.x, mc.y, mc.z, mc.w}, vw[4] = {vc.x, vc.y, vc.z, vc.w};
    float mmax = 0.0f, vmax = 0.0f;
    if (now.gscale != 1.0f) {                                  // (the same for all threads)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float2 x = __fmul2_rn(pair_of(g, q), make_float2(now.gscale, now.gscale));
            m[q] = x;
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) m[q] = pair_of(g, q);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float t[4];
        float2 u[2];
        e4m3x4_to_f32(mw[q], t);
        e4m4x4_to_f32(vw[q], u);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float2 x = m[2 * q + h];
            m[2 * q + h] = __fmul2_rn(make_float2(t[2 * h], t[2 * h + 1]), make_float2(sm, sm));
            v[2 * q + h] = __fmul2_rn(u[h], make_float2(sv, sv));
            adam_moments(s, x, m[2 * q + h], v[2 * q + h]);
            mmax = absmax3(mmax, m[2 * q + h].x, m[2 * q + h].y);
            vmax = absmax3(vmax, v[2 * q + h].x, v[2 * q + h].y);
        }
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) {                          // the block's eight lanes
        const float om = __shfl_xor_sync(0xFFFFFFFFu, mmax, d), ov = __shfl_xor_sync(0xFFFFFFFFu, vmax, d);
        mmax = absmax3(mmax, om, om);
        vmax = absmax3(vmax, ov, ov);
    }
    if (block_nonfinite(abs_word(mmax)) || block_nonfinite(abs_word(vmax))) {      // the block is left as it was
        note(s.status, SRQ_ERR_NONFINITE);
        return;
    }
    if (!FULL && left <= 0) return;
    const float im = block_inv(abs_word(mmax)), iv = e4m4_inv(vmax);
    uint32_t cm[4], cv[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (FULL) {                                  // the weights leave shared memory when they are due
            if (sizeof(P) == 4 || (q & 1) == 0) {
                constexpr int words = sizeof(P) == 4 ? 4 : 2;
                const uint4 x = b->piece[q * words / 4][lane];
                p.w[q * words] = x.x; p.w[q * words + 1] = x.y; p.w[q * words + 2] = x.z; p.w[q * words + 3] = x.w;
            }
        }
        uint32_t w[4], tv[4], tm[4];
        adam_words(s, ((uint64_t)i >> 2) + q, (uint32_t)id, (uint32_t)(id >> 32), w);
        // thresholds with half a unit below them, where they meet the bits below a code that stands in the top byte
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            tv[h] = __byte_perm(w[h], 0x80u, 0x5324);          // 0, upper half, 0x80
            tm[h] = tv[h] ^ __byte_perm(w[h], 0u, 0x5105);     // 0, upper ^ lower half, 0x80
        }
        const float2 m0 = m[2 * q], m1 = m[2 * q + 1], v0 = v[2 * q], v1 = v[2 * q + 1];
        uint2 x = code_bits(m0, im), y = code_bits(m1, im);
        // three bits of mantissa: code at bit 20; four: at bit 19.  The sign is shifted out and put back.
        const uint32_t mag = top_bytes((x.x << 4) + tm[0], (x.y << 4) + tm[1], (y.x << 4) + tm[2], (y.y << 4) + tm[3]);
        cm[q] = (mag & 0x7F7F7F7Fu) | (top_bytes(x.x, x.y, y.x, y.y) & 0x80808080u);
        x = code_bits(v0, iv); y = code_bits(v1, iv);
        uint32_t c = top_bytes((x.x << 5) + tv[0], (x.y << 5) + tv[1], (y.x << 5) + tv[2], (y.y << 5) + tv[3]);
        if (((c - 0x01010101u) & ~c & 0x80808080u) != 0 && iv > 0.0f) {          // a code is 0: a positive moment takes the next
            if ((c & 0x000000FFu) == 0 && v0.x > 0.0f) c |= 0x00000001u;
            if ((c & 0x0000FF00u) == 0 && v0.y > 0.0f) c |= 0x00000100u;
            if ((c & 0x00FF0000u) == 0 && v1.x > 0.0f) c |= 0x00010000u;
            if ((c & 0xFF000000u) == 0 && v1.y > 0.0f) c |= 0x01000000u;
        }
        cv[q] = c;
        const float2 a0 = adam_weight(s, now, pair_of(p, 2 * q), m0, v0), a1 = adam_weight(s, now, pair_of(p, 2 * q + 1), m1, v1);
        if constexpr (sizeof(P) == 2 && SR) {
            p.w[2 * q] = bf16_pair_sr(a0, w[0], w[1]);
            p.w[2 * q + 1] = bf16_pair_sr(a1, w[2], w[3]);
        } else if constexpr (sizeof(P) == 2) {
            p.w[2 * q] = bf16_pair(a0);
            p.w[2 * q + 1] = bf16_pair(a1);
        } else {
            p.w[4 * q] = __float_as_uint(a0.x); p.w[4 * q + 1] = __float_as_uint(a0.y);
            p.w[4 * q + 2] = __float_as_uint(a1.x); p.w[4 * q + 3] = __float_as_uint(a1.y);
        }
    }
    if (FULL) write16<P>(e.p, i, p, ((uintptr_t)e.p & 31u) == 0); else write_some<P>(e.p, i, p, left);
    write_codes(e.m, i, cm, left);
    write_codes(e.v, i, cv, left);
    if ((threadIdx.x & 7) == 0) { e.m_step[i / QBLK] = moment_step(mmax, im, 1.0f / E4M3_MAX); e.v_step[i / QBLK] = moment_step(vmax, iv, 1.0f / E4M4_MAX); }
}

template <typename P, typename G, bool SR, int CAP>
__global__ void __launch_bounds__(ADAM_THREADS<true>, 5) adamw8_kernel(const __grid_constant__ AdamParams<CAP> a) {
    pdl_enter();
    constexpr int WARPS = ADAM_THREADS<true> / 32, GROUP = ADAM_GROUP<true>;
    __shared__ Staged<P, G> buffers[WARPS][2];
    const AdamScalars& s = a.s;
    const AdamNow now = adam_now(s);
    if (now.refused) {
        if (threadIdx.x == 0 && blockIdx.x == 0) note(s.status, now.refused);
        return;
    }
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0);
    Staged<P, G>* b = buffers[warp];
    const int64_t size = (int64_t)a.run * WARPS;
    for (int64_t chunk = blockIdx.x * size; chunk < a.groups; chunk += gridDim.x * size) {
        const int64_t chunk_end = chunk + size < a.groups ? chunk + size : a.groups;
        // the chunk's groups, tensor by tensor: whole groups, the next one's bytes on their way while one is worked on, then the rest
        for (int64_t u = chunk; u < chunk_end;) {
            const int k = adam_find(a, u);
            const AdamEntry& e = a.e[k];
            const int64_t tensor_end = k + 1 < a.count ? a.e[k + 1].first : a.groups, end = tensor_end < chunk_end ? tensor_end : chunk_end;
            const int64_t whole = e.first + e.n / GROUP, whole_end = whole < end ? whole : end;
            const int mine = (int)(whole_end - u) - warp, turns = mine > 0 ? (mine + WARPS - 1) / WARPS : 0;
            const uint64_t id = (((uint64_t)s.id_hi << 32) | s.id_lo) + (uint64_t)k + ((uint64_t)now.t << 32);
            int64_t i = (u + warp - e.first) * GROUP + lane * 16;
            float sm = 0.0f, sv = 0.0f, next_sm = 0.0f, next_sv = 0.0f;
            if (turns > 0) {
                stage<P, G>(b[0], e, i, lane);
                sm = e.m_step[i / QBLK];
                sv = e.v_step[i / QBLK];
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll 1
            for (int t = 0; t < turns; ++t) {
                if (t + 1 < turns) {
                    const int64_t n = i + WARPS * GROUP;
                    stage<P, G>(b[(t + 1) & 1], e, n, lane);
                    next_sm = e.m_step[n / QBLK];
                    next_sv = e.v_step[n / QBLK];
                }
                asm volatile("cp.async.commit_group;\ncp.async.wait_group 1;" ::: "memory");
                adam8_group<P, G, SR, true>(s, now, e, i, id, sm, sv, &b[t & 1]);
                i += WARPS * GROUP;
                sm = next_sm; sv = next_sv;
            }
            if (whole_end < end && (int)(whole_end - u) % WARPS == warp) {     // the tensor's last group
                i = (whole_end - e.first) * GROUP + lane * 16;
                if (i < e.n) { sm = e.m_step[i / QBLK]; sv = e.v_step[i / QBLK]; }
                adam8_group<P, G, SR, false>(s, now, e, i, id, sm, sv, nullptr);
            }
            u = end;
        }
    }
}

template <int CAP>
static cudaError_t launch_adamw_cap(const AdamScalars& s, const srq_adamw_tensor_t* t, int n, int32_t p_dt, int32_t g_dt, bool state8, bool sr, cudaStream_t st) {
    static_assert(sizeof(AdamParams<CAP>) <= 32764, "parameters of a kernel");
    AdamParams<CAP> a;
    a.s = s;
    a.count = 0;
    a.groups = 0;
    const int64_t group = state8 ? ADAM_GROUP<true> : ADAM_GROUP<false>;
    for (int i = 0; i < n; ++i) {                              // empty tensors stay in the list: the position numbers the thresholds
        AdamEntry& e = a.e[a.count++];
        e.p = t[i].param; e.g = t[i].grad; e.m = t[i].m; e.v = t[i].v; e.m_step = t[i].m_step; e.v_step = t[i].v_step; e.n = t[i].n;
        e.first = a.groups;
        a.groups += (t[i].n + group - 1) / group;
    }
    if (a.groups == 0) return cudaSuccess;
    const int sms = sm_count();
    if (sms == 0) return cudaErrorUnknown;
    // few groups: one per warp, on as many SMs as there are (36 tensors of 2048: 6.5 -> 3.5 us)
    const int threads = state8 ? ADAM_THREADS<true> : ADAM_THREADS<false>;
    const int64_t warps = (int64_t)sms * (state8 ? 20 : 32);   // that run at a time
    a.run = a.groups >= 4 * warps * ADAM_RUN<true> && state8 ? ADAM_RUN<true> : a.groups > warps * ADAM_RUN<false> ? ADAM_RUN<false> : 1;
    const int64_t chunk = (int64_t)a.run * (threads / 32), want = (a.groups + chunk - 1) / chunk, most = (int64_t)sms * 32;
    const dim3 grid((unsigned)(want < most ? want : most)), block(threads);
    const bool pf = p_dt == SRQ_F32, gf = g_dt == SRQ_F32;
    typedef __nv_bfloat16 H;
    cudaError_t e;
#define SRQ_ADAM(kernel)                                                                                                                                      \
    (pf ? (gf ? launch_pdl(kernel<float, float, false, CAP>, grid, block, 0, st, a) : launch_pdl(kernel<float, H, false, CAP>, grid, block, 0, st, a))        \
     : sr ? (gf ? launch_pdl(kernel<H, float, true, CAP>, grid, block, 0, st, a) : launch_pdl(kernel<H, H, true, CAP>, grid, block, 0, st, a))                \
          : (gf ? launch_pdl(kernel<H, float, false, CAP>, grid, block, 0, st, a) : launch_pdl(kernel<H, H, false, CAP>, grid, block, 0, st, a)))
    e = state8 ? SRQ_ADAM(adamw8_kernel) : SRQ_ADAM(adamw_kernel);
#undef SRQ_ADAM
    count_launch();
    return e;
}

cudaError_t launch_adamw(const AdamwArgs& a, cudaStream_t st) {
    const srq_adamw_t& h = *a.h;
    AdamScalars s = {};
    s.beta1 = (float)h.beta1; s.keep1 = (float)(1.0 - h.beta1);
    s.beta2 = (float)h.beta2; s.keep2 = (float)(1.0 - h.beta2);
    s.eps = (float)h.eps; s.lr = (float)h.lr; s.weight_decay = (float)h.weight_decay;
    if (h.step_device) {
        s.inv_bias1 = (float)log(h.beta1); s.inv_root_bias2 = (float)log(h.beta2);
    } else {
        s.inv_bias1 = (float)(1.0 / -expm1((double)h.step * log(h.beta1)));
        s.inv_root_bias2 = (float)(1.0 / sqrt(-expm1((double)h.step * log(h.beta2))));
    }
    s.lr_device = h.lr_device; s.step_device = h.step_device; s.grad_scale = h.grad_scale; s.status = a.status; s.step = h.step;
    const PhiloxKeys keys = make_philox_keys(h.seed, 0);
    for (int r = 0; r < 10; ++r) { s.k0[r] = keys.k0[r]; s.k1[r] = keys.k1[r]; }
    // three sizes of the list: the parameters of a launch are copied by the host (30 KB of them: 6 us a call instead of 4)
    constexpr int FEW = 24, SOME = 96, MANY = 480;
    for (int64_t i = 0; i < a.count;) {
        const int64_t rest = a.count - i;
        const int n = (int)(rest < MANY ? rest : MANY);
        const uint64_t id = h.tensor_id + (uint64_t)i;
        s.id_lo = (uint32_t)id; s.id_hi = (uint32_t)(id >> 32);
        const cudaError_t e = n <= FEW ? launch_adamw_cap<FEW>(s, a.tensors + i, n, a.param_dt, a.grad_dt, a.state8, a.sr, st)
                            : n <= SOME ? launch_adamw_cap<SOME>(s, a.tensors + i, n, a.param_dt, a.grad_dt, a.state8, a.sr, st)
                                        : launch_adamw_cap<MANY>(s, a.tensors + i, n, a.param_dt, a.grad_dt, a.state8, a.sr, st);
        if (e != cudaSuccess) return e;
        i += n;
    }
    return cudaSuccess;
}

}  // namespace srq
