// C-ABI entry points of the block-scaled operators: argument checks and the empty cases.
#include "common.cuh"

using namespace srq;

namespace {

inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool known_dtype(srq_dtype_t dt) { return dt == SRQ_F32 || dt == SRQ_BF16; }
inline int64_t blocks_of(int64_t n) { return (n + 127) / 128; }
constexpr int64_t kMaxExtent = 0x7FFFFFFFll;           // tile coordinates are 32-bit

// A matrix with no elements may have null pointers (torch gives them to such tensors); its shape, pitches and modes are checked
// all the same.
inline bool empty(int64_t rows, int64_t cols) { return rows == 0 || cols == 0; }

// A [rows, cols] block-coded matrix.  any_tile: 128 x 128 tiles are allowed as well as 1 x 128 blocks.
srq_status_t check_blocks(const srq_blocks_t* b, int64_t rows, int64_t cols, bool any_tile) {
    if (!b || (!empty(rows, cols) && (!b->codes || !b->scale))) return SRQ_ERR_INVALID_ARG;
    if (b->tile_rows != 1 && b->tile_rows != 128) return SRQ_ERR_INVALID_ARG;
    if (b->tile_rows != 1 && !any_tile) return SRQ_ERR_UNSUPPORTED;
    if (rows > kMaxExtent || cols > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    if (!aligned_to(b->codes, 16) || b->ld % 16 != 0 || b->ld < cols) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(b->scale, 4) || b->ld_scale < blocks_of(cols)) return SRQ_ERR_INVALID_ARG;
    return SRQ_OK;
}
srq_status_t check_optional(const srq_blocks_t* b, int64_t rows, int64_t cols, bool any_tile) {
    return b ? check_blocks(b, rows, cols, any_tile) : SRQ_OK;
}

srq_status_t check_rounding(const srq_qspec_t* q, BlockRounding* r) {
    if (!q) return SRQ_ERR_INVALID_ARG;
    if (q->round != SRQ_SR && q->round != SRQ_RTN && q->round != SRQ_SR8 && q->round != SRQ_RNE) return SRQ_ERR_INVALID_ARG;
    if (q->scale != SRQ_PER_TENSOR && q->scale != SRQ_PER_ROW && q->scale != SRQ_PER_BLOCK) return SRQ_ERR_INVALID_ARG;
    if (q->format != SRQ_GRID_INT && q->format != SRQ_GRID_E4M3) return SRQ_ERR_INVALID_ARG;
    if (q->format != SRQ_GRID_E4M3 || q->bits != 8 || q->scale != SRQ_PER_BLOCK || (q->round != SRQ_SR && q->round != SRQ_RNE))
        return SRQ_ERR_UNSUPPORTED;
    r->sr = q->round == SRQ_SR;
    r->index_offset = q->index_offset; r->seed = q->seed; r->tensor_id = q->tensor_id;
    return SRQ_OK;
}

srq_status_t status_of(cudaError_t e) { return e == cudaSuccess ? SRQ_OK : SRQ_ERR_CUDA; }

#define SRQ_TRY(expr) do { const srq_status_t s_ = (expr); if (s_ != SRQ_OK) return s_; } while (0)

srq_status_t quantize_to(const BlockSource& src, const srq_qspec_t* q, const srq_blocks_t* rm, const srq_blocks_t* tr,
                         uint32_t* device_status, void* cuda_stream) {
    BlockRounding rnd;
    SRQ_TRY(check_rounding(q, &rnd));
    if (!rm && !tr) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_optional(rm, src.rows, src.cols, true));
    SRQ_TRY(check_optional(tr, src.cols, src.rows, true));
    if (!aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (src.rows > kMaxExtent || src.cols > kMaxExtent || blocks_of(src.rows) * blocks_of(src.cols) > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    if (empty(src.rows, src.cols)) return SRQ_OK;
    return status_of(launch_quantize_blocks(src, rnd, to_blocks(rm), to_blocks(tr), device_status, (cudaStream_t)cuda_stream));
}

}  // namespace

extern "C" {

srq_status_t srq_quantize_blocks(const void* x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld, const srq_qspec_t* q,
                                 const srq_blocks_t* rm, const srq_blocks_t* tr, uint32_t* device_status, void* cuda_stream) {
    if (rows < 0 || cols < 0 || ld < cols || !known_dtype(dt) || !aligned_to(x, 16)) return SRQ_ERR_INVALID_ARG;
    if (!x && !empty(rows, cols)) return SRQ_ERR_INVALID_ARG;
    BlockSource src;
    src.x = x; src.dt = dt; src.ld = ld; src.rows = rows; src.cols = cols;
    return quantize_to(src, q, rm, tr, device_status, cuda_stream);
}

srq_status_t srq_requantize_blocks(const srq_blocks_t* x, int64_t rows, int64_t cols, const srq_qspec_t* q, const srq_blocks_t* rm,
                                   const srq_blocks_t* tr, uint32_t* device_status, void* cuda_stream) {
    if (rows < 0 || cols < 0) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_blocks(x, rows, cols, true));
    BlockSource src;
    src.coded = to_blocks(x); src.rows = rows; src.cols = cols;
    return quantize_to(src, q, rm, tr, device_status, cuda_stream);
}

srq_status_t srq_gemm_blocks(const srq_blocks_t* a, const srq_blocks_t* b, int64_t M, int64_t N, int64_t Kc, void* out,
                             srq_dtype_t out_dt, int64_t ldo, int32_t accumulate, uint32_t* device_status, void* cuda_stream) {
    if (M < 0 || N < 0 || Kc < 0 || ldo < N || !known_dtype(out_dt)) return SRQ_ERR_INVALID_ARG;
    if (!out && !empty(M, N)) return SRQ_ERR_INVALID_ARG;
    if (accumulate != 0 && accumulate != 1) return SRQ_ERR_INVALID_ARG;
    if (accumulate && out_dt != SRQ_F32) return SRQ_ERR_UNSUPPORTED;      // running sums stay in binary32
    SRQ_TRY(check_blocks(a, M, Kc, true));
    SRQ_TRY(check_blocks(b, N, Kc, true));
    const size_t esize = out_dt == SRQ_BF16 ? 2 : 4;
    if (!aligned_to(out, esize) || !aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (empty(M, N)) return SRQ_OK;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (Kc == 0) {                                                        // empty contraction: the product is zero
        if (accumulate) return SRQ_OK;
        return status_of(cudaMemset2DAsync(out, (size_t)ldo * esize, 0, (size_t)N * esize, (size_t)M, st));
    }
    GemmBlocksArgs g;
    g.a = to_blocks(a); g.b = to_blocks(b); g.M = M; g.N = N; g.Kc = Kc;
    g.out = out; g.out_dt = out_dt; g.ldo = ldo; g.accumulate = accumulate;
    return launch_gemm_blocks(g, device_status, st);
}

srq_status_t srq_rmsnorm_fwd(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, srq_dtype_t dt,
                             const void* w, srq_dtype_t w_dt, int64_t rows, int64_t cols, float eps, const srq_qspec_t* q,
                             const srq_blocks_t* y, void* y_out, int64_t ld_y, void* r_out, int64_t ld_r, float* rstd,
                             uint32_t* device_status, void* cuda_stream) {
    if (rows < 0 || cols < 0 || !known_dtype(dt) || !known_dtype(w_dt) || !(eps >= 0.0f)) return SRQ_ERR_INVALID_ARG;
    if (!empty(rows, cols) && (!x || !w || (!y && !y_out))) return SRQ_ERR_INVALID_ARG;
    if (ldx < cols || (residual && ld_residual < cols) || (y_out && ld_y < cols) || (r_out && ld_r < cols)) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(x, 16) || !aligned_to(residual, 16) || !aligned_to(w, 16) || !aligned_to(y_out, 16) || !aligned_to(r_out, 16) ||
        !aligned_to(rstd, 4) || !aligned_to(device_status, 4))
        return SRQ_ERR_INVALID_ARG;
    NormFwdArgs a = {};
    if (y) {
        SRQ_TRY(check_rounding(q, &a.rnd));
        SRQ_TRY(check_blocks(y, rows, cols, false));
    }
    if (rows > kMaxExtent || cols > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    if (empty(rows, cols)) return SRQ_OK;
    a.x = x; a.ldx = ldx; a.residual = residual; a.ld_residual = ld_residual; a.dt = dt; a.w = w; a.w_dt = w_dt;
    a.rows = rows; a.cols = cols; a.eps = eps; a.y = to_blocks(y); a.y_out = y_out; a.ld_y = ld_y; a.r_out = r_out; a.ld_r = ld_r;
    a.rstd = rstd; a.status = device_status;
    return status_of(launch_rmsnorm_fwd(a, (cudaStream_t)cuda_stream));
}

size_t srq_rmsnorm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return 0;
    return rmsnorm_partial_bytes(rows, cols);
}

srq_status_t srq_rmsnorm_bwd(const void* dy, int64_t ld_dy, const void* r, int64_t ld_r, const void* d_residual, int64_t ld_dres,
                             srq_dtype_t dt, const void* w, srq_dtype_t w_dt, const float* rstd, int64_t rows, int64_t cols,
                             void* dx, int64_t ld_dx, float* dw, void* ws, size_t ws_bytes, void* cuda_stream) {
    if (rows < 0 || cols < 0 || !known_dtype(dt) || !known_dtype(w_dt)) return SRQ_ERR_INVALID_ARG;
    if (!empty(rows, cols) && (!dy || !r || !w || !rstd || (!dx && !dw))) return SRQ_ERR_INVALID_ARG;
    if (ld_dy < cols || ld_r < cols || (d_residual && ld_dres < cols) || (dx && ld_dx < cols)) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(dy, 16) || !aligned_to(r, 16) || !aligned_to(d_residual, 16) || !aligned_to(w, 16) || !aligned_to(dx, 16) ||
        !aligned_to(rstd, 4) || !aligned_to(dw, 4))
        return SRQ_ERR_INVALID_ARG;
    if (rows > kMaxExtent || cols > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    if (dw) {
        if (!ws || !aligned_to(ws, 256)) return SRQ_ERR_INVALID_ARG;
        if (ws_bytes < rmsnorm_partial_bytes(rows, cols)) return SRQ_ERR_WORKSPACE;
    }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cols == 0) return SRQ_OK;
    if (rows == 0) return dw ? status_of(cudaMemsetAsync(dw, 0, (size_t)cols * 4, st)) : SRQ_OK;
    NormBwdArgs a;
    a.dy = dy; a.ld_dy = ld_dy; a.r = r; a.ld_r = ld_r; a.d_residual = d_residual; a.ld_dres = ld_dres; a.dt = dt; a.w = w; a.w_dt = w_dt;
    a.rstd = rstd; a.rows = rows; a.cols = cols; a.dx = dx; a.ld_dx = ld_dx; a.dw = dw; a.partial = (float*)ws;
    return status_of(launch_rmsnorm_bwd(a, st));
}

srq_status_t srq_glu_fwd(const srq_blocks_t* x, const srq_blocks_t* wg, const srq_blocks_t* wu, int64_t T, int64_t F, int64_t K,
                         srq_act_t act, const srq_blocks_t* h, void* h_out, srq_dtype_t h_dt, int64_t ld_h,
                         const srq_blocks_t* gate, const srq_blocks_t* up, uint32_t* device_status, void* cuda_stream) {
    if (T < 0 || F < 0 || K <= 0 || (act != SRQ_SILU && act != SRQ_GELU)) return SRQ_ERR_INVALID_ARG;
    if (!empty(T, F) && !h && !h_out) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_blocks(x, T, K, true));
    SRQ_TRY(check_blocks(wg, F, K, true));
    SRQ_TRY(check_blocks(wu, F, K, true));
    if (wg->tile_rows != wu->tile_rows) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_optional(h, T, F, false));
    SRQ_TRY(check_optional(gate, T, F, false));
    SRQ_TRY(check_optional(up, T, F, false));
    if (h_out && (!known_dtype(h_dt) || ld_h < F || !aligned_to(h_out, 16))) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (empty(T, F)) return SRQ_OK;
    GluArgs g;
    g.x = to_blocks(x); g.wg = to_blocks(wg); g.wu = to_blocks(wu); g.T = T; g.F = F; g.K = K; g.act = act;
    g.h = to_blocks(h); g.gate = to_blocks(gate); g.up = to_blocks(up); g.h_out = h_out; g.h_dt = h_dt; g.ld_h = ld_h;
    return launch_glu_fwd(g, device_status, (cudaStream_t)cuda_stream);
}

srq_status_t srq_glu_bwd(const void* dh, srq_dtype_t dt, int64_t ld_dh, const srq_blocks_t* gate, const srq_blocks_t* up,
                         int64_t T, int64_t F, srq_act_t act, const srq_qspec_t* q, const srq_blocks_t* dg, const srq_blocks_t* du,
                         const srq_blocks_t* dg_t, const srq_blocks_t* du_t, const srq_blocks_t* h_t, uint32_t* device_status,
                         void* cuda_stream) {
    if (T < 0 || F < 0 || ld_dh < F || !known_dtype(dt) || !aligned_to(dh, 16)) return SRQ_ERR_INVALID_ARG;
    if (!dh && !empty(T, F)) return SRQ_ERR_INVALID_ARG;
    if (act != SRQ_SILU && act != SRQ_GELU) return SRQ_ERR_INVALID_ARG;
    BlockRounding rnd;
    SRQ_TRY(check_rounding(q, &rnd));
    SRQ_TRY(check_blocks(gate, T, F, false));
    SRQ_TRY(check_blocks(up, T, F, false));
    if (!dg && !du && !dg_t && !du_t && !h_t) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_optional(dg, T, F, false));
    SRQ_TRY(check_optional(du, T, F, false));
    SRQ_TRY(check_optional(dg_t, F, T, false));
    SRQ_TRY(check_optional(du_t, F, T, false));
    SRQ_TRY(check_optional(h_t, F, T, false));
    if (!aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (blocks_of(T) * blocks_of(F) > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    if (empty(T, F)) return SRQ_OK;
    return status_of(launch_glu_bwd(dh, dt, ld_dh, to_blocks(gate), to_blocks(up), T, F, act, rnd, to_blocks(dg), to_blocks(du),
                                    to_blocks(dg_t), to_blocks(du_t), to_blocks(h_t), device_status, (cudaStream_t)cuda_stream));
}

}  // extern "C"
