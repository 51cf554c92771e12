// AdamW step over many tensors at once (the formula and the formats of the 8-bit moments are in srq.h).
//
// The list of tensors travels in the kernel's parameters, so that a call needs no table on the device and can be recorded as it
// is.  Work is cut into groups of 256 elements of one tensor; a warp takes a group, a lane eight neighbouring elements of it, so
// that a block of 128 (the unit of an 8-bit moment's step size) is the sixteen lanes of half a warp: everything is read once,
// the block's new moments stay in registers between their absmax and their codes, and what is written is written once.
// 32-bit states are bound by HBM.  With 8-bit states and bfloat16 weights 10 bytes move per element while Philox takes about 20
// issue slots per 32 elements and the arithmetic and the packing about 40, which is near what HBM allows.
#include "train.cuh"

namespace srq {

constexpr int ADAM_GROUP = 256;                 // elements a warp takes at a time
constexpr int ADAM_THREADS = 256;

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
    int32_t count;
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

// 8-bit codes of the second moment (E4M4 without a sign).  Shifted to binary32's place of the exponent and multiplied by 2^120 a
// code is the number it stands for, subnormal ones included.
__device__ __forceinline__ float2 e4m4_pair(uint32_t a, uint32_t b) {
    const float2 up = make_float2(0x1p120f, 0x1p120f);
    return __fmul2_rn(make_float2(__uint_as_float(a & 0x07F80000u), __uint_as_float(b & 0x07F80000u)), up);
}
__device__ __forceinline__ void e4m4x8_to_f32(uint2 w, float2 v[4]) {
    v[0] = e4m4_pair(w.x << 19, w.x << 11); v[1] = e4m4_pair(w.x << 3, w.x >> 5);
    v[2] = e4m4_pair(w.y << 19, w.y << 11); v[3] = e4m4_pair(w.y << 3, w.y >> 5);
}
// |x| / D as a binary32 pattern whose exponent field is the code's (times 2^-120), plus the threshold below the code's last bit.
__device__ __forceinline__ uint32_t threshold_sum(float quotient, uint32_t threshold) {
    return (__float_as_uint(__fmul_rn(quotient, 0x1p-120f)) & 0x7FFFFFFFu) + threshold;
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
    bool go;
};
__device__ __forceinline__ AdamNow adam_now(const AdamScalars& s) {
    AdamNow n;
    float ib1 = s.inv_bias1, ib2 = s.inv_root_bias2;
    n.t = (uint32_t)s.step;
    if (s.step_device) {
        const int64_t t = *s.step_device;
        n.t = (uint32_t)t;
        // 1 - beta^t = -(e^(t ln beta) - 1): no cancellation for betas near 1
        ib1 = 1.0f / -expm1f((float)t * ib1);
        ib2 = 1.0f / sqrtf(-expm1f((float)t * ib2));
    }
    const float lr = s.lr_device ? *s.lr_device : s.lr;
    n.rate = lr * ib1;
    n.decay = 1.0f - lr * s.weight_decay;
    n.root = ib2;
    n.gscale = s.grad_scale ? *s.grad_scale : 1.0f;
    n.go = abs_word(n.gscale) < 0x7F800000u;
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
// bfloat16 by cutting off 16 bits after the threshold was added.  What is not finite stays so (a NaN keeps a payload bit).
__device__ __forceinline__ uint32_t bf16_sr_bits(float x, uint32_t u16) {
    const uint32_t b = __float_as_uint(x);
    return (b & 0x7FFFFFFFu) >= 0x7F800000u ? ((b & 0x7FFFFFFFu) > 0x7F800000u ? b | 0x00400000u : b) : b + u16;
}
__device__ __forceinline__ uint32_t bf16_pair(float2 x) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Philox words of the eight elements whose first has the flat index i (a multiple of 8).
__device__ __forceinline__ void adam_words(const AdamScalars& s, int64_t i, uint32_t c2, uint32_t c3, uint32_t w[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint64_t j = ((uint64_t)i >> 2) + h;
        uint32_t x0 = (uint32_t)j, x1 = (uint32_t)(j >> 32), x2 = c2, x3 = c3;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p0 = (uint64_t)0xD2511F53u * x0, p1 = (uint64_t)0xCD9E8D57u * x2;
            x0 = (uint32_t)(p1 >> 32) ^ x1 ^ s.k0[r];
            x1 = (uint32_t)p1;
            x2 = (uint32_t)(p0 >> 32) ^ x3 ^ s.k1[r];
            x3 = (uint32_t)p0;
        }
        w[4 * h] = x0; w[4 * h + 1] = x1; w[4 * h + 2] = x2; w[4 * h + 3] = x3;
    }
}

// P, G: types of weights and gradients.  SR: bfloat16 weights are rounded stochastically (8-bit moments always are).
template <typename P, typename G, bool STATE8, bool SR, int CAP>
__global__ void __launch_bounds__(ADAM_THREADS) adamw_kernel(const __grid_constant__ AdamParams<CAP> a) {
    pdl_enter();
    constexpr bool WORDS = STATE8 || (SR && sizeof(P) == 2);
    const AdamScalars& s = a.s;
    const AdamNow now = adam_now(s);
    if (!now.go) {
        if (threadIdx.x == 0 && blockIdx.x == 0) note(s.status, SRQ_ERR_NONFINITE);
        return;
    }
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (ADAM_THREADS / 32);
    for (int64_t u = (int64_t)blockIdx.x * (ADAM_THREADS / 32) + (threadIdx.x >> 5); u < a.groups; u += warps) {
        int k = 0;                                             // last tensor that begins at or before group u
        for (int hi = a.count; hi - k > 1;) {
            const int mid = (k + hi) >> 1;
            if (a.e[mid].first <= u) k = mid; else hi = mid;
        }
        const AdamEntry& e = a.e[k];
        const int64_t i = (u - e.first) * ADAM_GROUP + lane * 8;
        const int64_t left = e.n - i;                          // elements of this lane: min(left, 8), none or less: none
        float2 p[4], g[4], m[4], v[4];
        uint2 mc, vc;
        if (left >= 8) {
            read8<G>(e.g, i, g);
            read8<P>(e.p, i, p);
            if constexpr (STATE8) {
                mc = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(e.m) + i);
                vc = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(e.v) + i);
            } else {
                read8<float>(e.m, i, m);
                read8<float>(e.v, i, v);
            }
        } else {
            mc = make_uint2(0, 0); vc = make_uint2(0, 0);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float pp = 0.0f, gg = 0.0f, mm = 0.0f, vv = 0.0f;
                if (q < left) {
                    gg = read1<G>(e.g, i + q);
                    pp = read1<P>(e.p, i + q);
                    if constexpr (STATE8) {
                        const uint32_t cm = reinterpret_cast<const uint8_t*>(e.m)[i + q], cv = reinterpret_cast<const uint8_t*>(e.v)[i + q];
                        if (q < 4) { mc.x |= cm << (8 * q); vc.x |= cv << (8 * q); }
                        else { mc.y |= cm << (8 * q - 32); vc.y |= cv << (8 * q - 32); }
                    } else {
                        mm = read1<float>(e.m, i + q);
                        vv = read1<float>(e.v, i + q);
                    }
                }
                if (q & 1) { p[q >> 1].y = pp; g[q >> 1].y = gg; if constexpr (!STATE8) { m[q >> 1].y = mm; v[q >> 1].y = vv; } }
                else { p[q >> 1].x = pp; g[q >> 1].x = gg; if constexpr (!STATE8) { m[q >> 1].x = mm; v[q >> 1].x = vv; } }
            }
        }
        if constexpr (STATE8) {
            float sm = 0.0f, sv = 0.0f;
            if (left > 0) { sm = e.m_step[i / QBLK]; sv = e.v_step[i / QBLK]; }
            float t[4];
            e4m3x4_to_f32(mc.x, t); m[0] = make_float2(t[0], t[1]); m[1] = make_float2(t[2], t[3]);
            e4m3x4_to_f32(mc.y, t); m[2] = make_float2(t[0], t[1]); m[3] = make_float2(t[2], t[3]);
            e4m4x8_to_f32(vc, v);
#pragma unroll
            for (int q = 0; q < 4; ++q) { m[q] = __fmul2_rn(m[q], make_float2(sm, sm)); v[q] = __fmul2_rn(v[q], make_float2(sv, sv)); }
        }
        uint32_t w[8];
        if constexpr (WORDS) {
            const uint64_t id = (((uint64_t)s.id_hi << 32) | s.id_lo) + (uint64_t)k + ((uint64_t)now.t << 32);
            adam_words(s, i, (uint32_t)id, (uint32_t)(id >> 32), w);
        }
        float mmax = 0.0f, vmax = 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            g[q] = __fmul2_rn(g[q], make_float2(now.gscale, now.gscale));
            adam_moments(s, g[q], m[q], v[q]);
            mmax = absmax3(mmax, m[q].x, m[q].y);
            vmax = absmax3(vmax, v[q].x, v[q].y);
        }
        bool keep = true;
        if constexpr (STATE8) {
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) {                  // the block's sixteen lanes
                mmax = absmax3(mmax, mmax, __shfl_xor_sync(0xFFFFFFFFu, mmax, d));
                vmax = absmax3(vmax, vmax, __shfl_xor_sync(0xFFFFFFFFu, vmax, d));
            }
        }
        if (block_nonfinite(abs_word(mmax)) || block_nonfinite(abs_word(vmax))) {
            note(s.status, SRQ_ERR_NONFINITE);
            keep = !STATE8;
        }
        if (!keep || left <= 0) continue;
        uint32_t pb[8];                                        // weights: binary32 bits, or bfloat16 ones in the upper half
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 x = adam_weight(s, now, p[q], m[q], v[q]);
            if constexpr (sizeof(P) == 2 && SR) {
                pb[2 * q] = bf16_sr_bits(x.x, w[2 * q] & 0xFFFFu);
                pb[2 * q + 1] = bf16_sr_bits(x.y, w[2 * q + 1] & 0xFFFFu);
            } else if constexpr (sizeof(P) == 2) {
                const uint32_t b = bf16_pair(x);
                pb[2 * q] = b << 16; pb[2 * q + 1] = b & 0xFFFF0000u;
            } else {
                pb[2 * q] = __float_as_uint(x.x); pb[2 * q + 1] = __float_as_uint(x.y);
            }
        }
        if constexpr (STATE8) {
            const float im = block_inv(abs_word(mmax)), iv = e4m4_inv(vmax);
            uint32_t cm[8], cv[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float mm = q & 1 ? m[q >> 1].y : m[q >> 1].x, vv = q & 1 ? v[q >> 1].y : v[q >> 1].x;
                const uint32_t hi = w[q] >> 16, lo = w[q] & 0xFFFFu;
                cm[q] = (threshold_sum(__fmul_rn(mm, im), ((lo ^ hi) << 4) + 8u) >> 20) | ((__float_as_uint(mm) >> 24) & 0x80u);
                cv[q] = threshold_sum(__fmul_rn(vv, iv), (hi << 3) + 4u) >> 19;
                if (cv[q] == 0 && vv > 0.0f && iv > 0.0f) cv[q] = 1;
            }
            mc = make_uint2(cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24, cm[4] | cm[5] << 8 | cm[6] << 16 | cm[7] << 24);
            vc = make_uint2(cv[0] | cv[1] << 8 | cv[2] << 16 | cv[3] << 24, cv[4] | cv[5] << 8 | cv[6] << 16 | cv[7] << 24);
            if ((lane & 15) == 0) { e.m_step[i / QBLK] = moment_step(mmax, im, 1.0f / E4M3_MAX); e.v_step[i / QBLK] = moment_step(vmax, iv, 1.0f / E4M4_MAX); }
        }
        if (left >= 8) {
            if constexpr (sizeof(P) == 2) {
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(e.p) + i) =
                    make_uint4(__byte_perm(pb[0], pb[1], 0x7632), __byte_perm(pb[2], pb[3], 0x7632), __byte_perm(pb[4], pb[5], 0x7632), __byte_perm(pb[6], pb[7], 0x7632));
            } else {
                uint4* o = reinterpret_cast<uint4*>(reinterpret_cast<float*>(e.p) + i);
                o[0] = make_uint4(pb[0], pb[1], pb[2], pb[3]);
                o[1] = make_uint4(pb[4], pb[5], pb[6], pb[7]);
            }
            if constexpr (STATE8) {
                *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(e.m) + i) = mc;
                *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(e.v) + i) = vc;
            } else {
                write8(e.m, i, m);
                write8(e.v, i, v);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (q >= left) continue;
                if constexpr (sizeof(P) == 2) reinterpret_cast<uint16_t*>(e.p)[i + q] = (uint16_t)(pb[q] >> 16);
                else reinterpret_cast<uint32_t*>(e.p)[i + q] = pb[q];
                if constexpr (STATE8) {
                    reinterpret_cast<uint8_t*>(e.m)[i + q] = (uint8_t)((q < 4 ? mc.x : mc.y) >> (8 * (q & 3)));
                    reinterpret_cast<uint8_t*>(e.v)[i + q] = (uint8_t)((q < 4 ? vc.x : vc.y) >> (8 * (q & 3)));
                } else {
                    reinterpret_cast<float*>(e.m)[i + q] = q & 1 ? m[q >> 1].y : m[q >> 1].x;
                    reinterpret_cast<float*>(e.v)[i + q] = q & 1 ? v[q >> 1].y : v[q >> 1].x;
                }
            }
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
    for (int i = 0; i < n; ++i) {                              // empty tensors stay in the list: the position numbers the thresholds
        AdamEntry& e = a.e[a.count++];
        e.p = t[i].param; e.g = t[i].grad; e.m = t[i].m; e.v = t[i].v; e.m_step = t[i].m_step; e.v_step = t[i].v_step; e.n = t[i].n;
        e.first = a.groups;
        a.groups += (t[i].n + ADAM_GROUP - 1) / ADAM_GROUP;
    }
    if (a.groups == 0) return cudaSuccess;
    const int sms = sm_count();
    if (sms == 0) return cudaErrorUnknown;
    const int64_t want = (a.groups + ADAM_THREADS / 32 - 1) / (ADAM_THREADS / 32), most = (int64_t)sms * 32;
    const dim3 grid((unsigned)(want < most ? want : most)), block(ADAM_THREADS);
    const bool pf = p_dt == SRQ_F32, gf = g_dt == SRQ_F32;
    typedef __nv_bfloat16 H;
    cudaError_t e;
    if (state8) {
        if (pf) e = gf ? launch_pdl(adamw_kernel<float, float, true, true, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<float, H, true, true, CAP>, grid, block, 0, st, a);
        else if (sr) e = gf ? launch_pdl(adamw_kernel<H, float, true, true, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<H, H, true, true, CAP>, grid, block, 0, st, a);
        else e = gf ? launch_pdl(adamw_kernel<H, float, true, false, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<H, H, true, false, CAP>, grid, block, 0, st, a);
    } else {
        if (pf) e = gf ? launch_pdl(adamw_kernel<float, float, false, false, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<float, H, false, false, CAP>, grid, block, 0, st, a);
        else if (sr) e = gf ? launch_pdl(adamw_kernel<H, float, false, true, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<H, H, false, true, CAP>, grid, block, 0, st, a);
        else e = gf ? launch_pdl(adamw_kernel<H, float, false, false, CAP>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<H, H, false, false, CAP>, grid, block, 0, st, a);
    }
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
    constexpr int FEW = 24, MANY = 480;
    for (int64_t i = 0; i < a.count;) {
        const int64_t rest = a.count - i;
        const int n = (int)(rest < MANY ? rest : MANY);
        const uint64_t id = h.tensor_id + (uint64_t)i;
        s.id_lo = (uint32_t)id; s.id_hi = (uint32_t)(id >> 32);
        const cudaError_t e = n <= FEW ? launch_adamw_cap<FEW>(s, a.tensors + i, n, a.param_dt, a.grad_dt, a.state8, a.sr, st)
                                       : launch_adamw_cap<MANY>(s, a.tensors + i, n, a.param_dt, a.grad_dt, a.state8, a.sr, st);
        if (e != cudaSuccess) return e;
        i += n;
    }
    return cudaSuccess;
}

}  // namespace srq
