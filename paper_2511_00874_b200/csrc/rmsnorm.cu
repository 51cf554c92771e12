// Root-mean-square norm with the residual's addition and an output in block codes, and its backward pass.
//
// A row belongs to `tpr` threads (a power of two from 32 to 1024), a CTA to threads / tpr rows at a time.
// Thread t of a row holds the groups of eight columns t, t + tpr, ... (V of them) in registers, so that a
// row is read once: sum of squares (binary32, a fixed tree), then the norm, then the absmax of each
// 128-column block, which sits in 16 neighbouring lanes, then the codes.  Rows too long for the registers are
// walked again from memory (the LONG form).  Both passes are bound by HBM.
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

struct NormFwdParams {
    NormFwdArgs a;
    PhiloxKeys keys;
    int32_t tpr;                     // threads per row
    int32_t vec;                     // bit 0: x, 1: residual, 2: w, 3: r_out, 4: y_out allow 16-byte accesses
    int32_t rows_per_cta;
};

template <typename W>
__device__ __forceinline__ void load_w8(const void* w, int64_t c, int64_t cols, bool vec, float v[8]) { load8((const W*)w, c, cols, vec, v); }

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
            if constexpr (SR) thresholds8(a.rnd.index_offset + (uint64_t)row * (uint64_t)a.cols + (uint64_t)c, P.keys, rnd);
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
    const float rstd = __frcp_rn(__fsqrt_rn(__fadd_rn(__fdiv_rn(s, (float)a.cols), a.eps)));
    if (live && t == 0 && a.rstd) a.rstd[row] = rstd;
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
    int32_t tpr;
    int32_t vec;                     // bit 0: dy, 1: r, 2: d_residual, 3: w, 4: dx allow 16-byte accesses
    int32_t slots;                   // rows a CTA works on at a time
    int64_t partial_ld;
};

// Row `first`, first + step, ... of one slot: every thread keeps its columns, so that the weight's gradient adds
// up in its registers (or, for LONG rows, in its own words of the partial row) and leaves as one partial row
// per slot.
template <typename T, typename W, int V>
__global__ void __launch_bounds__(512) rmsnorm_bwd_kernel(const __grid_constant__ NormBwdParams P) {
    pdl_enter();
    __shared__ float red[2][32];
    const NormBwdArgs& a = P.a;
    const int tpr = P.tpr, t = threadIdx.x & (tpr - 1), slot = threadIdx.x / tpr;
    const int64_t first = (int64_t)blockIdx.x * P.slots + slot, step = (int64_t)gridDim.x * P.slots;
    float* part = a.dw ? a.partial + first * P.partial_ld : nullptr;
    const float inv_cols = 1.0f / (float)a.cols;
    float w[V ? V : 1][8], dw[V ? V : 1][8];
    if constexpr (V > 0) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            load8((const W*)a.w, ((int64_t)k * tpr + t) * 8, a.cols, P.vec & 8, w[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dw[k][e] = 0.0f;
        }
    } else if (part) {
        for (int64_t c = (int64_t)t * 8; c < a.cols; c += (int64_t)tpr * 8)
            for (int e = 0; e < 8; ++e) part[c + e] = 0.0f;            // partial rows are padded to whole groups
    }
    const int64_t rounds = (a.rows + step - 1) / step;                  // the same for every slot: barriers inside
    for (int64_t it = 0; it < rounds; ++it) {
        const int64_t row = first + it * step;
        const bool live = row < a.rows;
        const T* dy = (const T*)a.dy + row * a.ld_dy;
        const T* r = (const T*)a.r + row * a.ld_r;
        const float rstd = live ? a.rstd[row] : 0.0f;
        float g[V ? V : 1][8], n[V ? V : 1][8];
        auto load_row = [&](int64_t c, float gy[8], float nn[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) gy[e] = nn[e] = 0.0f;
            if (!live || c >= a.cols) return;
            load8(dy, c, a.cols, P.vec & 1, gy);
            load8(r, c, a.cols, P.vec & 2, nn);
#pragma unroll
            for (int e = 0; e < 8; ++e) nn[e] *= rstd;
        };
        float s = 0.0f;
        if constexpr (V > 0) {
#pragma unroll
            for (int k = 0; k < V; ++k) load_row(((int64_t)k * tpr + t) * 8, g[k], n[k]);
#pragma unroll
            for (int k = 0; k < V; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[k][e] = fmaf(g[k][e], n[k][e], dw[k][e]);
                    g[k][e] *= w[k][e];
                    s = fmaf(g[k][e], n[k][e], s);
                }
            }
        } else {
            for (int64_t c = (int64_t)t * 8; c < a.cols; c += (int64_t)tpr * 8) {
                load_row(c, g[0], n[0]);
                load8((const W*)a.w, c, a.cols, P.vec & 8, w[0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (part) part[c + e] = fmaf(g[0][e], n[0][e], part[c + e]);
                    s = fmaf(g[0][e] * w[0][e], n[0][e], s);
                }
            }
        }
        s = row_sum(s, tpr, red[it & 1]) * inv_cols;
        if (a.dx && live) {
            auto finish = [&](int64_t c, const float gw[8], const float nn[8]) {
                if (c >= a.cols) return;
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = rstd * fmaf(-nn[e], s, gw[e]);
                if (a.d_residual) {
                    float q[8];
                    load8((const T*)a.d_residual + row * a.ld_dres, c, a.cols, P.vec & 4, q);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] += q[e];
                }
                store8((T*)a.dx + row * a.ld_dx, c, a.cols, P.vec & 16, o);
            };
            if constexpr (V > 0) {
#pragma unroll
                for (int k = 0; k < V; ++k) finish(((int64_t)k * tpr + t) * 8, g[k], n[k]);
            } else {
                for (int64_t c = (int64_t)t * 8; c < a.cols; c += (int64_t)tpr * 8) {
                    load_row(c, g[0], n[0]);
                    load8((const W*)a.w, c, a.cols, P.vec & 8, w[0]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[0][e] *= w[0][e];
                    finish(c, g[0], n[0]);
                }
            }
        }
    }
    if constexpr (V > 0) {
        if (part) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int64_t c = ((int64_t)k * tpr + t) * 8;
                if (c < P.partial_ld) {
                    *reinterpret_cast<float4*>(part + c) = make_float4(dw[k][0], dw[k][1], dw[k][2], dw[k][3]);
                    *reinterpret_cast<float4*>(part + c + 4) = make_float4(dw[k][4], dw[k][5], dw[k][6], dw[k][7]);
                }
            }
        }
    }
}

// dw[c] = sum of the partial rows, in a fixed order: 8 warps take every eighth row of 32 columns, then one adds up.
__global__ void __launch_bounds__(256) rmsnorm_dw_kernel(const float* __restrict__ partial, int64_t n, int64_t ld, int64_t cols,
                                                         float* __restrict__ dw) {
    pdl_enter();
    __shared__ float part[8][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < cols)
        for (int64_t r = warp; r < n; r += 8) s += partial[r * ld + c];
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < cols) {
        for (int i = 1; i < 8; ++i) s += part[i][lane];
        dw[c] = s;
    }
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static bool vec16(const void* p, int64_t ld, int32_t dt) { return (uintptr_t)p % 16 == 0 && ld % (dt == SRQ_F32 ? 4 : 8) == 0; }

// Threads per row and groups per thread for rows of `groups` groups of eight: V as small as 1024 threads allow
// when there are few rows (latency), else about two to four groups per thread (fewer threads to meet).
// v_max: 4 at most; V = 0: the row does not fit.
static void row_shape(int64_t groups, bool few, int max_threads, int* tpr, int* v) {
    int want = few ? 1 : 2;
    int p = 32;
    while (p < max_threads && (int64_t)p * want < groups) p <<= 1;
    *tpr = p;
    const int64_t need = (groups + p - 1) / p;
    *v = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 0;
}

template <typename T, typename W, bool SR>
static cudaError_t launch_fwd(const NormFwdParams& P, int v, dim3 grid, dim3 block, cudaStream_t st) {
    switch (v) {
        case 1: return launch_pdl(rmsnorm_fwd_kernel<T, W, 1, SR>, grid, block, 0, st, P);
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
    int v;
    row_shape((a.cols + 7) / 8, a.rows < 512, 1024, &P.tpr, &v);
    const int threads = P.tpr < 256 ? 256 : P.tpr;
    P.rows_per_cta = threads / P.tpr;
    const dim3 grid((unsigned)((a.rows + P.rows_per_cta - 1) / P.rows_per_cta)), block(threads);
    const bool f = a.dt == SRQ_F32, wf = a.w_dt == SRQ_F32;
    cudaError_t e;
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
static cudaError_t launch_bwd(const NormBwdParams& P, int v, dim3 grid, dim3 block, cudaStream_t st) {
    switch (v) {
        case 1: return launch_pdl(rmsnorm_bwd_kernel<T, W, 1>, grid, block, 0, st, P);
        case 2: return launch_pdl(rmsnorm_bwd_kernel<T, W, 2>, grid, block, 0, st, P);
        case 4: return launch_pdl(rmsnorm_bwd_kernel<T, W, 4>, grid, block, 0, st, P);
        default: return launch_pdl(rmsnorm_bwd_kernel<T, W, 0>, grid, block, 0, st, P);
    }
}

cudaError_t launch_rmsnorm_bwd(const NormBwdArgs& a, cudaStream_t stream) {
    NormBwdParams P;
    P.a = a;
    P.vec = (vec16(a.dy, a.ld_dy, a.dt) ? 1 : 0) | (vec16(a.r, a.ld_r, a.dt) ? 2 : 0) | (vec16(a.d_residual, a.ld_dres, a.dt) ? 4 : 0) |
            (vec16(a.w, 0, a.w_dt) ? 8 : 0) | (vec16(a.dx, a.ld_dx, a.dt) ? 16 : 0);
    P.partial_ld = pad64(a.cols);
    int v;
    row_shape((a.cols + 7) / 8, true, 512, &P.tpr, &v);
    // every slot leaves a partial row: at most as many as the workspace holds
    const int64_t n_max = a.rows < NORM_MAX_PARTIALS ? a.rows : NORM_MAX_PARTIALS;
    int slots = 256 / P.tpr;
    if (slots < 1) slots = 1;
    while (slots > 1 && slots > n_max) slots >>= 1;
    P.slots = slots;
    const int64_t ctas = n_max / slots;
    const dim3 grid((unsigned)ctas), block(slots * P.tpr);
    const bool f = a.dt == SRQ_F32, wf = a.w_dt == SRQ_F32;
    cudaError_t e;
    if (f) e = wf ? launch_bwd<float, float>(P, v, grid, block, stream) : launch_bwd<float, __nv_bfloat16>(P, v, grid, block, stream);
    else e = wf ? launch_bwd<__nv_bfloat16, float>(P, v, grid, block, stream) : launch_bwd<__nv_bfloat16, __nv_bfloat16>(P, v, grid, block, stream);
    count_launch();
    if (e != cudaSuccess || !a.dw) return e;
    e = launch_pdl(rmsnorm_dw_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(256), 0, stream, (const float*)a.partial,
                   ctas * slots, P.partial_ld, a.cols, a.dw);
    count_launch();
    return e;
}

}  // namespace srq
