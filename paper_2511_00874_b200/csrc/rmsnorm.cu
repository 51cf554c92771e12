// Root-mean-square norm with the residual's addition and an output in block codes, and its backward pass.
//
// A row belongs to `tpr` threads (a power of two from 32 to 1024), a CTA to threads / tpr rows at a time.
// Thread t of a row holds the groups of eight columns t, t + tpr, ... (V of them) in registers, so that a
// row is read once: sum of squares (binary32, a fixed tree), then the norm, then the absmax of each
// 128-column block, which sits in 16 neighbouring lanes, then the codes.  Both passes are bound by HBM.
//
// Three forms of each kernel.
//   stream   whole groups of eight columns, 16-byte aligned rows of at most 16384 elements (8192 backward), rounding to
//            nearest: walks rows with a grid of resident CTAs, keeps the weight in registers, has the next row's loads
//            in flight while a row is worked on, and works on two values per instruction
//   any      any extent up to 8192 and any pitch, rounding to nearest: a warp takes 128 columns at a time, a lane every 32nd of
//            them, so that rows that start anywhere are read in whole lines; the number of threads per row is a
//            compile-time constant, so that a lane's columns are immediate offsets (with eight neighbouring columns
//            per thread and bounds in 64 bits a value took 106 instructions and 2.5 times as long)
//   long     what is left: longer rows (V = 0: read twice), stochastic rounding
#include <mutex>

#include "blocks.cuh"

namespace srq {

constexpr int NORM_MAX_PARTIALS = 512;

struct NormShared { float red[32]; };

// Sum over the tpr threads of a row; every thread of the CTA takes part.  buf: 32 floats per use, two uses
// in turn so that one barrier suffices.
__device__ __forceinline__ float row_sum(float s, int tpr, float* buf) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (tpr == 32) return s;
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) buf[warp] = s;
    __syncthreads();
    const int wpr = tpr >> 5, first = warp / wpr * wpr;
    float t = 0.0f;
    for (int i = 0; i < wpr; ++i) t += buf[first + i];
    return t;
}

// 1 / sqrt(mean + eps) from a row's sum of squares: the fast approximation and one Newton step (x (1.5 - 0.5 m x^2), the
// correction in one fused operation), within about one unit of the last place.
__device__ __forceinline__ float rstd_of(float sum, float inv_cols, float eps) {
    const float m = fmaf(sum, inv_cols, eps);
    float x;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(x) : "f"(m));
    if (!(m > 1e-30f && m < 1e30f)) return x;            // zero, tiny, huge: nothing to gain, much to overflow
    return fmaf(x * 0.5f, fmaf(-m * x, x, 1.0f), x);
}

// One thread per row: stores 1 / rms and reports a row for which it is no positive finite number (the mean square is NaN or
// overflows binary32, or is 0 where eps is), since a row of finite values would leave as zeros without a trace.
__device__ __forceinline__ void finish_rstd(const NormFwdArgs& a, int64_t row, float rstd) {
    if (a.rstd) a.rstd[row] = rstd;
    if (!(rstd > 0.0f && rstd < __int_as_float(0x7F800000))) note(a.status, SRQ_ERR_NONFINITE);
}

// Eight values of a row as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<float> { uint4 a, b; };
template <> struct Raw8<__nv_bfloat16> { uint4 a; };
__device__ __forceinline__ void load_raw(Raw8<float>& q, const float* p) {
    q.a = __ldcs(reinterpret_cast<const uint4*>(p)); q.b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
}
__device__ __forceinline__ void load_raw(Raw8<__nv_bfloat16>& q, const __nv_bfloat16* p) { q.a = __ldcs(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void zero_raw(Raw8<float>& q) { q.a = q.b = make_uint4(0u, 0u, 0u, 0u); }
__device__ __forceinline__ void zero_raw(Raw8<__nv_bfloat16>& q) { q.a = make_uint4(0u, 0u, 0u, 0u); }
__device__ __forceinline__ float2 f2(uint32_t x, uint32_t y) { return make_float2(__uint_as_float(x), __uint_as_float(y)); }
__device__ __forceinline__ float2 bf2(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ void widen(const Raw8<float>& q, float2 (&v)[4]) { v[0] = f2(q.a.x, q.a.y); v[1] = f2(q.a.z, q.a.w); v[2] = f2(q.b.x, q.b.y); v[3] = f2(q.b.z, q.b.w); }
__device__ __forceinline__ void widen(const Raw8<__nv_bfloat16>& q, float2 (&v)[4]) { v[0] = bf2(q.a.x); v[1] = bf2(q.a.y); v[2] = bf2(q.a.z); v[3] = bf2(q.a.w); }
__device__ __forceinline__ uint32_t bf16x2_of(float2 v) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ void store_narrow(float* p, const float2 (&v)[4]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
__device__ __forceinline__ void store_narrow(__nv_bfloat16* p, const float2 (&v)[4]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16x2_of(v[0]), bf16x2_of(v[1]), bf16x2_of(v[2]), bf16x2_of(v[3]));
}
__device__ __forceinline__ float absmax8(const float2 (&v)[4]) {
    return absmax3(absmax3(v[0].x, v[0].y, v[1].x), absmax3(v[1].y, v[2].x, v[2].y), absmax3(v[3].x, v[3].y, 0.0f));
}

struct NormFwdParams {
    NormFwdArgs a;
    PhiloxKeys keys;
    int32_t tpr;                     // threads per row
    int32_t vec;                     // bit 0: x, 1: residual, 2: w, 3: r_out, 4: y_out allow 16-byte accesses
    int32_t rows_per_cta;
    float inv_cols;
};

template <typename T, typename W, int V>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512) rmsnorm_fwd_stream_kernel(const __grid_constant__ NormFwdParams P) {
    pdl_enter();
    __shared__ float red[2][32];
    const NormFwdArgs& a = P.a;
    const int tpr = P.tpr, t = threadIdx.x & (tpr - 1), slot = threadIdx.x / tpr, lane = threadIdx.x & 31;
    const int64_t step = (int64_t)gridDim.x * P.rows_per_cta;
    const int32_t cols = (int32_t)a.cols, c0 = t * 8, dc = tpr * 8;      // this thread's groups: c0, c0 + dc, ...
    Raw8<W> w[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (c0 + k * dc < cols) load_raw(w[k], (const W*)a.w + c0 + k * dc); else zero_raw(w[k]);
    Raw8<T> nx[V], nr[V];
    auto fetch = [&](int64_t row) {
        const T* x = (const T*)a.x + row * a.ldx + c0;
        const T* q = (const T*)a.residual + row * a.ld_residual + c0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            zero_raw(nx[k]); zero_raw(nr[k]);
            if (row < a.rows && c0 + k * dc < cols) {
                load_raw(nx[k], x + k * dc);
                if (a.residual) load_raw(nr[k], q + k * dc);
            }
        }
    };
    int64_t row = (int64_t)blockIdx.x * P.rows_per_cta + slot;
    fetch(row);
    const int64_t rounds = (a.rows + step - 1) / step;                  // the same for every row of the CTA: barriers inside
#pragma unroll 1
    for (int64_t it = 0; it < rounds; ++it, row += step) {
        const bool live = row < a.rows;
        float2 v[V][4], s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            widen(nx[k], v[k]);
            if (a.residual) {
                float2 q[4];
                widen(nr[k], q);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = __fadd2_rn(v[k][e], q[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s2 = __ffma2_rn(v[k][e], v[k][e], s2);
        }
        if (it + 1 < rounds) fetch(row + step);
        const float rstd = rstd_of(row_sum(s2.x + s2.y, tpr, red[it & 1]), P.inv_cols, a.eps);
        if (live && t == 0) finish_rstd(a, row, rstd);
        const float2 rs2 = make_float2(rstd, rstd);
        uint32_t m[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int32_t c = c0 + k * dc;
            const bool in = live && c < cols;
            if (in && a.r_out) store_narrow((T*)a.r_out + row * a.ld_r + c, v[k]);
            float2 ww[4];
            widen(w[k], ww);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k][e] = __fmul2_rn(__fmul2_rn(v[k][e], rs2), ww[e]);
            if (in && a.y_out) store_narrow((T*)a.y_out + row * a.ld_y + c, v[k]);
            m[k] = abs_word(absmax8(v[k]));
        }
        if (!a.y.codes) continue;
        // absmax of V blocks over 16 lanes: halve the blocks, then the lanes; lane l ends with block l % V's
#pragma unroll
        for (int b = 1; b < V; b <<= 1) {
            const bool odd = (lane & b) != 0;
#pragma unroll
            for (int i = 0; i < V / (2 * b); ++i) {
                const uint32_t keep = odd ? m[2 * i + 1] : m[2 * i], give = odd ? m[2 * i] : m[2 * i + 1];
                m[i] = max(keep, __shfl_xor_sync(0xFFFFFFFFu, give, b));
            }
        }
#pragma unroll
        for (int b = V; b < 16; b <<= 1) m[0] = max(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], b));
        const float inv = block_inv(m[0]);
        const int mine = lane & (V - 1);
        const int32_t c_mine = (c0 & ~(QBLK - 1)) + mine * dc;          // first column of the block this lane speaks for
        if (live && (lane & 15) < V && c_mine < cols) {
            a.y.scale[row * a.y.ld_scale + c_mine / QBLK] = block_size(m[0]);
            if (block_nonfinite(m[0])) note(a.status, SRQ_ERR_NONFINITE);
        }
        uint8_t* codes = a.y.codes + row * a.y.ld;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float f = V == 1 ? inv : __shfl_sync(0xFFFFFFFFu, inv, (lane & 16) + k);
            const int32_t c = c0 + k * dc;
            const uint32_t lo = encode4<false>(v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y, f, f, f, f, 0, 0, 0, 0);
            const uint32_t hi = encode4<false>(v[k][2].x, v[k][2].y, v[k][3].x, v[k][3].y, f, f, f, f, 0, 0, 0, 0);
            if (live && c < cols) *reinterpret_cast<uint2*>(codes + c) = make_uint2(lo, hi);
        }
    }
}

template <typename W>
__device__ __forceinline__ void load_w8(const void* w, int64_t c, int64_t cols, bool vec, float v[8]) { load8((const W*)w, c, cols, vec, v); }

// The columns of lane `lane` of warp `warp` of a row in the any form: first + column_offset<TPR>(e), e = 0 .. 4 KB - 1.
template <int TPR> __device__ __forceinline__ constexpr int column_offset(int e) { return (e >> 2) * (TPR * 4) + (e & 3) * 32; }

template <typename T, typename W, int TPR, int KB>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rmsnorm_fwd_any_kernel(const __grid_constant__ NormFwdParams P) {
    pdl_enter();
    __shared__ float red[2][32];
    constexpr int E = 4 * KB;
    const NormFwdArgs& a = P.a;
    const int t = threadIdx.x & (TPR - 1), slot = threadIdx.x / TPR, lane = threadIdx.x & 31;
    const int32_t first = (t >> 5) * QBLK + lane, left = (int32_t)a.cols - first;      // column e exists: column_offset(e) < left
    const int64_t step = (int64_t)gridDim.x * P.rows_per_cta;
    float w[E];
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = column_offset<TPR>(e) < left ? (float)((const W*)a.w)[first + column_offset<TPR>(e)] : 0.0f;
    T nx[E], nq[E];
    auto fetch = [&](int64_t row) {
        const T* x = (const T*)a.x + row * a.ldx + first;
        const T* q = (const T*)a.residual + row * a.ld_residual + first;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = row < a.rows && column_offset<TPR>(e) < left;
            nx[e] = in ? x[column_offset<TPR>(e)] : (T)0.0f;
            nq[e] = in && a.residual ? q[column_offset<TPR>(e)] : (T)0.0f;
        }
    };
    int64_t row = (int64_t)blockIdx.x * P.rows_per_cta + slot;
    fetch(row);
    const int64_t rounds = (a.rows + step - 1) / step;
#pragma unroll 1
    for (int64_t it = 0; it < rounds; ++it, row += step) {
        const bool live = row < a.rows;
        float v[E], s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = __fadd_rn((float)nx[e], (float)nq[e]);
            s = fmaf(v[e], v[e], s);
        }
        if (it + 1 < rounds) fetch(row + step);
        const float rstd = rstd_of(row_sum(s, TPR, red[it & 1]), P.inv_cols, a.eps);
        if (!live) continue;                               // whole warps; the next barrier is the next row's
        if (t == 0) finish_rstd(a, row, rstd);
        if (a.r_out) {
            T* o = (T*)a.r_out + row * a.ld_r + first;
#pragma unroll
            for (int e = 0; e < E; ++e) if (column_offset<TPR>(e) < left) o[column_offset<TPR>(e)] = (T)v[e];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = v[e] * rstd * w[e];
        if (a.y_out) {
            T* o = (T*)a.y_out + row * a.ld_y + first;
#pragma unroll
            for (int e = 0; e < E; ++e) if (column_offset<TPR>(e) < left) o[column_offset<TPR>(e)] = (T)v[e];
        }
        if (!a.y.codes) continue;
        uint32_t m[KB], mine = 0u;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            m[k] = __reduce_max_sync(0xFFFFFFFFu, abs_word(absmax3(absmax3(v[4 * k], v[4 * k + 1], v[4 * k + 2]), v[4 * k + 3], 0.0f)));
            mine = (lane & (KB - 1)) == k ? m[k] : mine;   // lane k has the divisions of block k
        }
        const float inv = block_inv(mine);
        const int32_t block = (t >> 5) + lane * (TPR / 32);
        if (lane < KB && (int64_t)block * QBLK < a.cols) {
            a.y.scale[row * a.y.ld_scale + block] = block_size(mine);
            if (block_nonfinite(mine)) note(a.status, SRQ_ERR_NONFINITE);
        }
        uint8_t* codes = a.y.codes + row * a.y.ld + first;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            const float f = __shfl_sync(0xFFFFFFFFu, inv, k);
            const uint32_t c = encode4<false>(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3], f, f, f, f, 0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (column_offset<TPR>(4 * k + i) < left) codes[column_offset<TPR>(4 * k + i)] = (uint8_t)(c >> (8 * i));
        }
    }
}

// One group of eight of y: block codes and / or y itself.  All 32 lanes of the warp call it together; the
// sixteen lanes of a block have the same row and neighbouring groups.
template <typename T, bool SR>
__device__ __forceinline__ void norm_emit(const NormFwdParams& P, int64_t row, int64_t c, const float y[8]) {
    const NormFwdArgs& a = P.a;
    const bool in = row < a.rows && c < a.cols;
    if (a.y.codes) {
        uint32_t m = abs_word(absmax3(absmax3(y[0], y[1], y[2]), absmax3(y[3], y[4], y[5]), absmax3(y[6], y[7], 0.0f)));
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));
        float step, inv;
        block_step(m, &step, &inv);
        if (in) {
            if (block_nonfinite(m)) note(a.status, SRQ_ERR_NONFINITE);
            if ((c & (QBLK - 1)) == 0) a.y.scale[row * a.y.ld_scale + c / QBLK] = step;
            uint32_t rnd[8] = {};
            if constexpr (SR) thresholds8(a.rnd.index_offset + (uint64_t)row * (uint64_t)a.cols + (uint64_t)c, P.keys, step_word(a.rnd.step), rnd);
            const uint32_t lo = encode4<SR>(y[0], y[1], y[2], y[3], inv, inv, inv, inv, rnd[0], rnd[1], rnd[2], rnd[3]);
            const uint32_t hi = encode4<SR>(y[4], y[5], y[6], y[7], inv, inv, inv, inv, rnd[4], rnd[5], rnd[6], rnd[7]);
            store_codes8(a.y.codes + row * a.y.ld, c, a.cols, lo, hi);
        }
    }
    if (in && a.y_out) store8((T*)a.y_out + row * a.ld_y, c, a.cols, P.vec & 16, y);
}

// V groups per thread; V == 0: the row is read from memory twice.
template <typename T, typename W, int V, bool SR>
__global__ void __launch_bounds__(1024) rmsnorm_fwd_kernel(const __grid_constant__ NormFwdParams P) {
    pdl_enter();
    __shared__ NormShared S;
    const NormFwdArgs& a = P.a;
    const int tpr = P.tpr, t = threadIdx.x & (tpr - 1), slot = threadIdx.x / tpr;
    const int64_t row = (int64_t)blockIdx.x * P.rows_per_cta + slot;
    const bool live = row < a.rows;
    const T* x = (const T*)a.x + row * a.ldx;
    const T* res = a.residual ? (const T*)a.residual + row * a.ld_residual : nullptr;
    auto load_r = [&](int64_t c, float r[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = 0.0f;
        if (!live || c >= a.cols) return;
        load8(x, c, a.cols, P.vec & 1, r);
        if (res) {
            float q[8];
            load8(res, c, a.cols, P.vec & 2, q);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = __fadd_rn(r[e], q[e]);
        }
    };
    float keep[V ? V : 1][8];
    float s = 0.0f;
    if constexpr (V > 0) {
#pragma unroll
        for (int k = 0; k < V; ++k) load_r(((int64_t)k * tpr + t) * 8, keep[k]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(keep[k][e], keep[k][e], s);
        }
    } else {
        for (int64_t c = (int64_t)t * 8; c < a.cols; c += (int64_t)tpr * 8) {
            load_r(c, keep[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(keep[0][e], keep[0][e], s);
        }
    }
    s = row_sum(s, tpr, S.red);
    const float rstd = rstd_of(s, P.inv_cols, a.eps);
    if (live && t == 0) finish_rstd(a, row, rstd);
    auto finish = [&](int64_t c, const float r[8]) {
        if (live && a.r_out) store8((T*)a.r_out + row * a.ld_r, c, a.cols, P.vec & 8, r);
        float w[8], y[8];
        load_w8<W>(a.w, c, a.cols, P.vec & 4, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = r[e] * rstd * w[e];
        norm_emit<T, SR>(P, row, c, y);
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int k = 0; k < V; ++k) finish(((int64_t)k * tpr + t) * 8, keep[k]);
    } else {
        // whole warps stay in the loop: the lanes of a block exchange their maxima
        for (int64_t c = (int64_t)t * 8; c - (threadIdx.x & 31) * 8 < a.cols; c += (int64_t)tpr * 8) {
            load_r(c, keep[0]);
            finish(c, keep[0]);
        }
    }
}

struct NormBwdParams {
    NormBwdArgs a;
    float inv_cols;
    int32_t tpr;
    int32_t vec;                     // bit 0: dy, 1: r, 2: d_residual, 3: w, 4: dx allow 16-byte accesses
    int32_t slots;                   // rows a CTA works on at a time
    int64_t partial_ld;
};

// The streaming form; the slots of a CTA add up their shares of the weight's gradient through shared memory, so that there is
// one partial row per CTA.
template <typename T, typename W, int V>
__global__ void __launch_bounds__(512) rmsnorm_bwd_stream_kernel(const __grid_constant__ NormBwdParams P) {
    pdl_enter();
    extern __shared__ float4 share[];
    __shared__ float red[2][32];
    const NormBwdArgs& a = P.a;
    const int tpr = P.tpr, t = threadIdx.x & (tpr - 1), slot = threadIdx.x / tpr;
    const int64_t step = (int64_t)gridDim.x * P.slots;
    const int32_t cols = (int32_t)a.cols, c0 = t * 8, dc = tpr * 8;
    Raw8<W> w[V];
    float2 dw[V][4];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (c0 + k * dc < cols) load_raw(w[k], (const W*)a.w + c0 + k * dc); else zero_raw(w[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[k][e] = make_float2(0.0f, 0.0f);
    }
    Raw8<T> ny[V], nr[V];
    float next_rstd = 0.0f;
    auto fetch = [&](int64_t row) {
        const T* y = (const T*)a.dy + row * a.ld_dy + c0;
        const T* r = (const T*)a.r + row * a.ld_r + c0;
        next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            zero_raw(ny[k]); zero_raw(nr[k]);
            if (row < a.rows && c0 + k * dc < cols) { load_raw(ny[k], y + k * dc); load_raw(nr[k], r + k * dc); }
        }
    };
    int64_t row = (int64_t)blockIdx.x * P.slots + slot;
    fetch(row);
    const int64_t rounds = (a.rows + step - 1) / step;
#pragma unroll 1
    for (int64_t it = 0; it < rounds; ++it, row += step) {
        const bool live = row < a.rows;
        const float rstd = next_rstd;
        const float2 rs2 = make_float2(rstd, rstd);
        float2 g[V][4], n[V][4], s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float2 ww[4];
            widen(ny[k], g[k]);
            widen(nr[k], n[k]);
            widen(w[k], ww);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                n[k][e] = __fmul2_rn(n[k][e], rs2);
                dw[k][e] = __ffma2_rn(g[k][e], n[k][e], dw[k][e]);
                g[k][e] = __fmul2_rn(g[k][e], ww[e]);
                s2 = __ffma2_rn(g[k][e], n[k][e], s2);
            }
        }
        Raw8<T> q[V];                                                  // arrives while the row's sum is formed
        if (a.dx && a.d_residual) {
            const T* d = (const T*)a.d_residual + row * a.ld_dres + c0;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                zero_raw(q[k]);
                if (live && c0 + k * dc < cols) load_raw(q[k], d + k * dc);
            }
        }
        if (it + 1 < rounds) fetch(row + step);
        const float s = -row_sum(s2.x + s2.y, tpr, red[it & 1]) * P.inv_cols;
        if (!a.dx || !live) continue;
        const float2 m2 = make_float2(s, s);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int32_t c = c0 + k * dc;
            if (c >= cols) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) g[k][e] = __fmul2_rn(rs2, __ffma2_rn(n[k][e], m2, g[k][e]));
            if (a.d_residual) {
                float2 d[4];
                widen(q[k], d);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[k][e] = __fadd2_rn(g[k][e], d[e]);
            }
            store_narrow((T*)a.dx + row * a.ld_dx + c, g[k]);
        }
    }
    if (!a.dw) return;
    // slots 1, 2, ... hand their sums to slot 0, in this order
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (slot > 0) {
            share[((slot - 1) * V + k) * tpr * 2 + 2 * t] = make_float4(dw[k][0].x, dw[k][0].y, dw[k][1].x, dw[k][1].y);
            share[((slot - 1) * V + k) * tpr * 2 + 2 * t + 1] = make_float4(dw[k][2].x, dw[k][2].y, dw[k][3].x, dw[k][3].y);
        }
    }
    __syncthreads();
    if (slot > 0) return;
    float* part = a.partial + (int64_t)blockIdx.x * P.partial_ld;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int32_t c = c0 + k * dc;
        if (c >= P.partial_ld) continue;
        float4 x = make_float4(dw[k][0].x, dw[k][0].y, dw[k][1].x, dw[k][1].y), y = make_float4(dw[k][2].x, dw[k][2].y, dw[k][3].x, dw[k][3].y);
        for (int o = 0; o + 1 < P.slots; ++o) {
            const float4 p = share[(o * V + k) * tpr * 2 + 2 * t], q = share[(o * V + k) * tpr * 2 + 2 * t + 1];
            x.x += p.x; x.y += p.y; x.z += p.z; x.w += p.w;
            y.x += q.x; y.y += q.y; y.z += q.z; y.w += q.w;
        }
        reinterpret_cast<float4*>(part + c)[0] = x;
        reinterpret_cast<float4*>(part + c)[1] = y;
    }
}

template <typename T, typename W, int TPR, int KB>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rmsnorm_bwd_any_kernel(const __grid_constant__ NormBwdParams P) {
    pdl_enter();
    constexpr int E = 4 * KB, SLOTS = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[2][32];
    __shared__ float share[SLOTS > 1 ? SLOTS - 1 : 1][SLOTS > 1 ? E * TPR : 1];
    const NormBwdArgs& a = P.a;
    const int t = threadIdx.x & (TPR - 1), slot = threadIdx.x / TPR, lane = threadIdx.x & 31;
    const int32_t first = (t >> 5) * QBLK + lane, left = (int32_t)a.cols - first;
    const int64_t step = (int64_t)gridDim.x * SLOTS;
    float w[E], dw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        w[e] = column_offset<TPR>(e) < left ? (float)((const W*)a.w)[first + column_offset<TPR>(e)] : 0.0f;
        dw[e] = 0.0f;
    }
    T ny[E], nr[E];
    float next_rstd = 0.0f;
    auto fetch = [&](int64_t row) {
        const T* y = (const T*)a.dy + row * a.ld_dy + first;
        const T* r = (const T*)a.r + row * a.ld_r + first;
        next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = row < a.rows && column_offset<TPR>(e) < left;
            ny[e] = in ? y[column_offset<TPR>(e)] : (T)0.0f;
            nr[e] = in ? r[column_offset<TPR>(e)] : (T)0.0f;
        }
    };
    int64_t row = (int64_t)blockIdx.x * SLOTS + slot;
    fetch(row);
    const int64_t rounds = (a.rows + step - 1) / step;
#pragma unroll 1
    for (int64_t it = 0; it < rounds; ++it, row += step) {
        const bool live = row < a.rows;
        const float rstd = next_rstd;
        float g[E], n[E], s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            n[e] = (float)nr[e] * rstd;
            g[e] = (float)ny[e];
            dw[e] = fmaf(g[e], n[e], dw[e]);
            g[e] *= w[e];
            s = fmaf(g[e], n[e], s);
        }
        T q[E];
        if (a.dx && a.d_residual) {
            const T* d = (const T*)a.d_residual + row * a.ld_dres + first;
#pragma unroll
            for (int e = 0; e < E; ++e) q[e] = live && column_offset<TPR>(e) < left ? d[column_offset<TPR>(e)] : (T)0.0f;
        }
        if (it + 1 < rounds) fetch(row + step);
        s = -row_sum(s, TPR, red[it & 1]) * P.inv_cols;
        if (!a.dx || !live) continue;
        T* o = (T*)a.dx + row * a.ld_dx + first;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float x = rstd * fmaf(n[e], s, g[e]);
            if (a.d_residual) x += (float)q[e];
            if (column_offset<TPR>(e) < left) o[column_offset<TPR>(e)] = (T)x;
        }
    }
    if (!a.dw) return;
    // slots 1, 2, ... hand their sums to slot 0, in this order
    if constexpr (SLOTS > 1) {
        if (slot > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) share[slot - 1][e * TPR + t] = dw[e];
        }
        __syncthreads();
        if (slot > 0) return;
        for (int o = 0; o + 1 < SLOTS; ++o) {
#pragma unroll
            for (int e = 0; e < E; ++e) dw[e] += share[o][e * TPR + t];
        }
    }
    float* part = a.partial + (int64_t)blockIdx.x * P.partial_ld + first;
#pragma unroll
    for (int e = 0; e < E; ++e) if (column_offset<TPR>(e) < left) part[column_offset<TPR>(e)] = dw[e];
}

// Rows too long for the registers: read twice, one CTA of 512 threads per row at a time; the weight's gradient adds up in the
// CTA's own partial row.
template <typename T, typename W>
__global__ void __launch_bounds__(512) rmsnorm_bwd_long_kernel(const __grid_constant__ NormBwdParams P) {
    pdl_enter();
    __shared__ float red[2][32];
    const NormBwdArgs& a = P.a;
    const W* w = (const W*)a.w;
    float* part = a.dw ? a.partial + (int64_t)blockIdx.x * P.partial_ld : nullptr;
    if (part)
        for (int64_t c = threadIdx.x; c < a.cols; c += 512) part[c] = 0.0f;
    int use = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, use ^= 1) {
        const T* dy = (const T*)a.dy + row * a.ld_dy;
        const T* r = (const T*)a.r + row * a.ld_r;
        const float rstd = a.rstd[row];
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += 512) {
            const float gy = (float)dy[c], nn = (float)r[c] * rstd;
            if (part) part[c] = fmaf(gy, nn, part[c]);
            s = fmaf(gy * (float)w[c], nn, s);
        }
        s = row_sum(s, 512, red[use]) * P.inv_cols;
        if (!a.dx) continue;
        for (int64_t c = threadIdx.x; c < a.cols; c += 512) {
            const float d = a.d_residual ? (float)((const T*)a.d_residual)[row * a.ld_dres + c] : 0.0f;
            ((T*)a.dx)[row * a.ld_dx + c] = (T)(rstd * fmaf(-(float)r[c] * rstd, s, (float)dy[c] * (float)w[c]) + d);
        }
    }
}

// dw[c] = sum of the partial rows, in a fixed order: 32 warps take every 32nd row of 32 columns (at most sixteen rows each, all
// loads in flight at once), then one adds up.
__global__ void __launch_bounds__(1024) rmsnorm_dw_kernel(const float* __restrict__ partial, int64_t n, int64_t ld, int64_t cols,
                                                          float* __restrict__ dw) {
    pdl_enter();
    __shared__ float part[32][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float v[NORM_MAX_PARTIALS / 32], s = 0.0f;
#pragma unroll
    for (int i = 0; i < NORM_MAX_PARTIALS / 32; ++i) v[i] = (c < cols && warp + 32 * i < n) ? __ldcg(partial + (int64_t)(warp + 32 * i) * ld + c) : 0.0f;
#pragma unroll
    for (int i = 0; i < NORM_MAX_PARTIALS / 32; ++i) s += v[i];
    part[warp][lane] = s;
    __syncthreads();
    // warp w adds up column w
    s = part[lane][warp];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    const int64_t cw = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && cw < cols) dw[cw] = s;
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static bool vec16(const void* p, int64_t ld, int32_t dt) { return (uintptr_t)p % 16 == 0 && ld % (dt == SRQ_F32 ? 4 : 8) == 0; }

// Long form: threads per row (at most max_threads) and groups per thread for rows of `groups` groups of eight: V as small as the
// threads allow when there are few rows (latency), else two to four groups per thread (fewer threads to meet).  V = 0:
// the row does not fit four groups per thread.
static void row_shape(int64_t groups, bool few, int max_threads, int* tpr, int* v) {
    int want = few ? 1 : 2;
    int p = 32;
    while (p < max_threads && (int64_t)p * want < groups) p <<= 1;
    *tpr = p;
    const int64_t need = (groups + p - 1) / p;
    *v = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 0;
}

static int norm_sms() {
    static int sms[64] = {};
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    std::lock_guard<std::mutex> lock(mu);
    if (sms[dev] == 0 && cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms[dev];
}

// Streaming form: threads per row (groups of eight columns over V per thread) and rows per CTA of `threads` threads.
// v: groups per thread, 4 where rows are plentiful (the row's fixed work is shared by more values), fewer when a few rows
// are all there is (latency).
static void stream_shape(int64_t groups, int v_want, int threads, int* tpr, int* v, int* slots) {
    *v = v_want;
    while (*v > 1 && groups * 2 <= (int64_t)32 * *v) *v >>= 1;           // short rows: a warp need not hold empty groups
    int p = 32;
    while ((int64_t)p * *v < groups && p < 1024) p <<= 1;
    *tpr = p;
    *slots = p >= threads ? 1 : threads / p;
}

template <typename T, typename W>
static cudaError_t launch_fwd_stream(const NormFwdParams& P, int v, dim3 grid, dim3 block, cudaStream_t st) {
    switch (v) {
        case 1: return launch_pdl(rmsnorm_fwd_stream_kernel<T, W, 1>, grid, block, 0, st, P);
        case 2: return launch_pdl(rmsnorm_fwd_stream_kernel<T, W, 2>, grid, block, 0, st, P);
        default: return launch_pdl(rmsnorm_fwd_stream_kernel<T, W, 4>, grid, block, 0, st, P);
    }
}

// The any form: threads per row and blocks of 128 columns per warp for `cols` columns (at most 8192).
template <template <int, int> class Launch, typename... A>
static cudaError_t any_form(int64_t cols, A&&... args) {
    if (cols <= 256) return Launch<32, 2>::go(args...);
    if (cols <= 512) return Launch<32, 4>::go(args...);
    if (cols <= 1024) return Launch<128, 2>::go(args...);
    if (cols <= 2048) return Launch<128, 4>::go(args...);
    if (cols <= 4096) return Launch<512, 2>::go(args...);
    return Launch<512, 4>::go(args...);
}
// Resident CTAs of `threads` threads and at most 128 registers, or one per group of rows.
static unsigned any_grid(int64_t rows, int slots, int threads, int sms) {
    const int64_t want = (rows + slots - 1) / slots, most = (int64_t)sms * (threads <= 256 ? 2 : 1);
    return (unsigned)(want < most ? want : most);
}
template <typename T, typename W> struct FwdAny {
    template <int TPR, int KB> struct L {
        static cudaError_t go(NormFwdParams& P, int sms, cudaStream_t st) {
            constexpr int threads = TPR < 256 ? 256 : TPR;
            P.tpr = TPR; P.rows_per_cta = threads / TPR;
            return launch_pdl(rmsnorm_fwd_any_kernel<T, W, TPR, KB>, dim3(any_grid(P.a.rows, threads / TPR, threads, sms)), dim3(threads), 0, st, P);
        }
    };
};
template <typename T, typename W> struct BwdAny {
    template <int TPR, int KB> struct L {
        static cudaError_t go(NormBwdParams& P, int sms, unsigned* grid, cudaStream_t st) {
            constexpr int threads = TPR < 256 ? 256 : TPR;
            const unsigned n = any_grid(P.a.rows, threads / TPR, threads, sms);
            *grid = n < NORM_MAX_PARTIALS ? n : NORM_MAX_PARTIALS;
            return launch_pdl(rmsnorm_bwd_any_kernel<T, W, TPR, KB>, dim3(*grid), dim3(threads), 0, st, P);
        }
    };
};

template <typename T, typename W, bool SR>
static cudaError_t launch_fwd(const NormFwdParams& P, int v, dim3 grid, dim3 block, cudaStream_t st) {
    if constexpr (SR)                                          // rounded to nearest such short rows take the any form
        if (v == 1) return launch_pdl(rmsnorm_fwd_kernel<T, W, 1, SR>, grid, block, 0, st, P);
    switch (v) {
        case 2: return launch_pdl(rmsnorm_fwd_kernel<T, W, 2, SR>, grid, block, 0, st, P);
        case 4: return launch_pdl(rmsnorm_fwd_kernel<T, W, 4, SR>, grid, block, 0, st, P);
        default: return launch_pdl(rmsnorm_fwd_kernel<T, W, 0, SR>, grid, block, 0, st, P);
    }
}

cudaError_t launch_rmsnorm_fwd(const NormFwdArgs& a, cudaStream_t stream) {
    NormFwdParams P;
    P.a = a;
    P.keys = make_philox_keys(a.rnd.seed, a.rnd.tensor_id);
    P.vec = (vec16(a.x, a.ldx, a.dt) ? 1 : 0) | (vec16(a.residual, a.ld_residual, a.dt) ? 2 : 0) | (vec16(a.w, 0, a.w_dt) ? 4 : 0) |
            (vec16(a.r_out, a.ld_r, a.dt) ? 8 : 0) | (vec16(a.y_out, a.ld_y, a.dt) ? 16 : 0);
    P.inv_cols = 1.0f / (float)a.cols;
    int v;
    const bool f = a.dt == SRQ_F32, wf = a.w_dt == SRQ_F32;
    cudaError_t e;
    const bool aligned = (P.vec & 1) && (!a.residual || (P.vec & 2)) && (P.vec & 4) && (!a.r_out || (P.vec & 8)) && (!a.y_out || (P.vec & 16));
    const int sms = norm_sms();
    if (sms == 0) return cudaErrorUnknown;
    if (aligned && a.cols % 8 == 0 && !a.rnd.sr) {
        // few rows: as many threads on each as there are groups; else groups of four (two in binary32, whose values take twice
        // the registers)
        const bool few = a.rows <= sms;
        stream_shape(a.cols / 8, few ? 1 : f ? 2 : 4, few ? 32 : 256, &P.tpr, &v, &P.rows_per_cta);
        // rows that two groups per thread only hold with 1024 threads (binary32, over 8192 columns) take four too: the registers
        // for more than one group allow 512 threads.  4096 x 12288 with a residual 194 -> 173 us against the long form, x 8200
        // 165 -> 151, without a residual, or of 16384 columns, within 1.5 % of it, and 300 rows (two rounds and four rows) 18.1 -> 19.6.
        if ((int64_t)P.tpr * v * 8 < a.cols || (v > 1 && P.tpr > 512)) stream_shape(a.cols / 8, 4, 256, &P.tpr, &v, &P.rows_per_cta);
        const int threads = P.tpr * P.rows_per_cta;
        if ((int64_t)P.tpr * v * 8 >= a.cols && (v == 1 || threads <= 512)) {
            const int64_t want = (a.rows + P.rows_per_cta - 1) / P.rows_per_cta, most = (int64_t)sms * (threads <= 256 ? 2 : 1);
            const dim3 grid((unsigned)(want < most ? want : most)), block(threads);
            if (f) e = wf ? launch_fwd_stream<float, float>(P, v, grid, block, stream) : launch_fwd_stream<float, __nv_bfloat16>(P, v, grid, block, stream);
            else e = wf ? launch_fwd_stream<__nv_bfloat16, float>(P, v, grid, block, stream) : launch_fwd_stream<__nv_bfloat16, __nv_bfloat16>(P, v, grid, block, stream);
            count_launch();
            return e;
        }
    }
    if (a.cols <= 8192 && !a.rnd.sr) {
        if (f) e = wf ? any_form<FwdAny<float, float>::L>(a.cols, P, sms, stream) : any_form<FwdAny<float, __nv_bfloat16>::L>(a.cols, P, sms, stream);
        else e = wf ? any_form<FwdAny<__nv_bfloat16, float>::L>(a.cols, P, sms, stream) : any_form<FwdAny<__nv_bfloat16, __nv_bfloat16>::L>(a.cols, P, sms, stream);
        count_launch();
        return e;
    }
    row_shape((a.cols + 7) / 8, a.rows < 512, 1024, &P.tpr, &v);
    const int threads = P.tpr < 256 ? 256 : P.tpr;
    P.rows_per_cta = threads / P.tpr;
    const dim3 grid((unsigned)((a.rows + P.rows_per_cta - 1) / P.rows_per_cta)), block(threads);
#define SRQ_NORM(T, W) (a.rnd.sr ? launch_fwd<T, W, true>(P, v, grid, block, stream) : launch_fwd<T, W, false>(P, v, grid, block, stream))
    if (f) e = wf ? SRQ_NORM(float, float) : SRQ_NORM(float, __nv_bfloat16);
    else e = wf ? SRQ_NORM(__nv_bfloat16, float) : SRQ_NORM(__nv_bfloat16, __nv_bfloat16);
#undef SRQ_NORM
    count_launch();
    return e;
}

static int64_t pad64(int64_t n) { return (n + 63) / 64 * 64; }
size_t rmsnorm_partial_bytes(int64_t rows, int64_t cols) {
    const int64_t n = rows < 1 ? 1 : rows < NORM_MAX_PARTIALS ? rows : NORM_MAX_PARTIALS;
    return (size_t)n * pad64(cols) * 4;
}

template <typename T, typename W>
static cudaError_t launch_bwd_stream(const NormBwdParams& P, int v, dim3 grid, dim3 block, size_t smem, cudaStream_t st) {
    return v == 1 ? launch_pdl(rmsnorm_bwd_stream_kernel<T, W, 1>, grid, block, smem, st, P) : launch_pdl(rmsnorm_bwd_stream_kernel<T, W, 2>, grid, block, smem, st, P);
}
static cudaError_t launch_dw(const NormBwdArgs& a, int64_t partial_ld, int64_t n, cudaStream_t stream) {
    const cudaError_t e = launch_pdl(rmsnorm_dw_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(1024), 0, stream, (const float*)a.partial, n,
                                     partial_ld, a.cols, a.dw);
    count_launch();
    return e;
}

cudaError_t launch_rmsnorm_bwd(const NormBwdArgs& a, cudaStream_t stream) {
    NormBwdParams P;
    P.a = a;
    P.vec = (vec16(a.dy, a.ld_dy, a.dt) ? 1 : 0) | (vec16(a.r, a.ld_r, a.dt) ? 2 : 0) | (vec16(a.d_residual, a.ld_dres, a.dt) ? 4 : 0) |
            (vec16(a.w, 0, a.w_dt) ? 8 : 0) | (vec16(a.dx, a.ld_dx, a.dt) ? 16 : 0);
    P.partial_ld = pad64(a.cols);
    P.inv_cols = 1.0f / (float)a.cols;
    int v;
    const bool f = a.dt == SRQ_F32, wf = a.w_dt == SRQ_F32;
    cudaError_t e;
    const int sms = norm_sms();
    if (sms == 0) return cudaErrorUnknown;
    const bool aligned = (P.vec & 1) && (P.vec & 2) && (!a.d_residual || (P.vec & 4)) && (P.vec & 8) && (!a.dx || (P.vec & 16));
    if (aligned && a.cols % 8 == 0 && a.cols <= 512 * 2 * 8) {
        stream_shape(a.cols / 8, 2, 256, &P.tpr, &v, &P.slots);
        const int64_t want = (a.rows + P.slots - 1) / P.slots, most = (int64_t)sms * (P.tpr * P.slots <= 256 ? 2 : 1);
        const int64_t ctas = want < most ? want : most;            // one partial row each: at most 512 on any device
        const dim3 grid((unsigned)(ctas < NORM_MAX_PARTIALS ? ctas : NORM_MAX_PARTIALS)), block(P.tpr * P.slots);
        const size_t smem = (size_t)(P.slots - 1) * P.tpr * v * 32;
        if (f) e = wf ? launch_bwd_stream<float, float>(P, v, grid, block, smem, stream) : launch_bwd_stream<float, __nv_bfloat16>(P, v, grid, block, smem, stream);
        else e = wf ? launch_bwd_stream<__nv_bfloat16, float>(P, v, grid, block, smem, stream) : launch_bwd_stream<__nv_bfloat16, __nv_bfloat16>(P, v, grid, block, smem, stream);
        count_launch();
        if (e != cudaSuccess || !a.dw) return e;
        return launch_dw(a, P.partial_ld, grid.x, stream);
    }
    unsigned grid = 0;
    if (a.cols <= 8192) {
        if (f) e = wf ? any_form<BwdAny<float, float>::L>(a.cols, P, sms, &grid, stream) : any_form<BwdAny<float, __nv_bfloat16>::L>(a.cols, P, sms, &grid, stream);
        else e = wf ? any_form<BwdAny<__nv_bfloat16, float>::L>(a.cols, P, sms, &grid, stream) : any_form<BwdAny<__nv_bfloat16, __nv_bfloat16>::L>(a.cols, P, sms, &grid, stream);
    } else {
        grid = (unsigned)(a.rows < NORM_MAX_PARTIALS ? a.rows : NORM_MAX_PARTIALS);
        if (f) e = wf ? launch_pdl(rmsnorm_bwd_long_kernel<float, float>, dim3(grid), dim3(512), 0, stream, P) : launch_pdl(rmsnorm_bwd_long_kernel<float, __nv_bfloat16>, dim3(grid), dim3(512), 0, stream, P);
        else e = wf ? launch_pdl(rmsnorm_bwd_long_kernel<__nv_bfloat16, float>, dim3(grid), dim3(512), 0, stream, P) : launch_pdl(rmsnorm_bwd_long_kernel<__nv_bfloat16, __nv_bfloat16>, dim3(grid), dim3(512), 0, stream, P);
    }
    count_launch();
    if (e != cudaSuccess || !a.dw) return e;
    return launch_dw(a, P.partial_ld, grid, stream);
}

}  // namespace srq
