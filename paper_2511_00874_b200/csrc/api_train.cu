// C-ABI entry points of the operators at the ends of a training step: argument checks and the empty cases.
#include <math.h>

#include "common.cuh"

using namespace srq;

namespace {

inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool known_dtype(srq_dtype_t dt) { return dt == SRQ_F32 || dt == SRQ_BF16; }
inline bool known_index(srq_index_t t) { return t == SRQ_I32 || t == SRQ_I64; }
inline size_t index_bytes(srq_index_t t) { return t == SRQ_I64 ? 8 : 4; }
inline bool empty(int64_t rows, int64_t cols) { return rows == 0 || cols == 0; }
inline srq_status_t status_of(cudaError_t e) { return e == cudaSuccess ? SRQ_OK : SRQ_ERR_CUDA; }
constexpr int64_t kMaxExtent = 0x7FFFFFFEll;           // rows, tokens and classes are counted in 32 bits
constexpr int64_t kMaxColumns = 1ll << 20;             // of an embedding: a grid's second extent

#define SRQ_TRY(expr) do { const srq_status_t s_ = (expr); if (s_ != SRQ_OK) return s_; } while (0)

// A matrix of logits with its targets; one without elements may have null pointers.
srq_status_t check_logits(const void* x, srq_dtype_t dt, int64_t rows, int64_t classes, int64_t ld, const void* targets, srq_index_t target_t,
                          float temperature, const uint32_t* status) {
    if (rows < 0 || classes < 0 || !known_dtype(dt) || !known_index(target_t) || !(temperature >= 0x1p-100f && temperature <= 0x1p100f)) return SRQ_ERR_INVALID_ARG;
    if ((!x && !empty(rows, classes)) || (!targets && rows)) return SRQ_ERR_INVALID_ARG;
    if (ld < classes || !aligned_to(x, 16) || !aligned_to(targets, index_bytes(target_t)) || !aligned_to(status, 4)) return SRQ_ERR_INVALID_ARG;
    if (rows > kMaxExtent || classes > kMaxExtent) return SRQ_ERR_UNSUPPORTED;
    return SRQ_OK;
}
// The gradient's matrix: its own memory, or the logits' (same pointer, then the same pitch).
srq_status_t check_dlogits(const void* x, int64_t ld, const void* dx, int64_t ldx, int64_t classes) {
    if (!dx) return SRQ_OK;
    if (!aligned_to(dx, 16) || ldx < classes || (dx == x && ldx != ld)) return SRQ_ERR_INVALID_ARG;
    return SRQ_OK;
}

}  // namespace

extern "C" {

srq_status_t srq_embedding_fwd(const void* table, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld, const void* ids, srq_index_t id_t, int64_t tokens,
                               float scale, void* out, srq_dtype_t out_dt, int64_t ld_out, uint32_t* device_status, void* cuda_stream) {
    if (rows < 0 || cols < 0 || tokens < 0 || ld < cols || ld_out < cols || !known_dtype(dt) || !known_dtype(out_dt) || !known_index(id_t)) return SRQ_ERR_INVALID_ARG;
    if ((!table && !empty(rows, cols)) || (!ids && tokens) || (!out && !empty(tokens, cols))) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(table, 16) || !aligned_to(out, 16) || !aligned_to(ids, index_bytes(id_t)) || !aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (rows > kMaxExtent || tokens > kMaxExtent || cols > kMaxColumns) return SRQ_ERR_UNSUPPORTED;
    if (empty(tokens, cols)) return SRQ_OK;
    const EmbedFwdArgs a = {table, dt, rows, cols, ld, ids, id_t, tokens, scale, out, out_dt, ld_out, device_status};
    return status_of(launch_embedding_fwd(a, (cudaStream_t)cuda_stream));
}

size_t srq_embedding_workspace_bytes(int64_t tokens, int64_t rows, int64_t cols) {
    if (tokens < 0 || rows < 0 || cols < 0 || tokens > kMaxExtent || rows > kMaxExtent || cols > kMaxColumns) return 0;
    return embedding_bytes(tokens, cols);
}

srq_status_t srq_embedding_bwd(const void* dout, srq_dtype_t dt, int64_t tokens, int64_t cols, int64_t ld, const void* ids, srq_index_t id_t, int64_t rows,
                               float scale, void* dtable, srq_dtype_t dtable_dt, int64_t ld_dtable, int32_t accumulate, void* ws, size_t ws_bytes,
                               uint32_t* device_status, void* cuda_stream) {
    if (rows < 0 || cols < 0 || tokens < 0 || ld < cols || ld_dtable < cols || !known_dtype(dt) || !known_dtype(dtable_dt) || !known_index(id_t))
        return SRQ_ERR_INVALID_ARG;
    if (accumulate != 0 && accumulate != 1) return SRQ_ERR_INVALID_ARG;
    if (accumulate && dtable_dt != SRQ_F32) return SRQ_ERR_UNSUPPORTED;   // running sums stay in binary32
    if ((!dout && !empty(tokens, cols)) || (!ids && tokens) || (!dtable && !empty(rows, cols))) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(dout, 16) || !aligned_to(dtable, 16) || !aligned_to(ids, index_bytes(id_t)) || !aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    if (rows > kMaxExtent || tokens > kMaxExtent || cols > kMaxColumns) return SRQ_ERR_UNSUPPORTED;
    if (!ws || !aligned_to(ws, 256)) return SRQ_ERR_INVALID_ARG;
    if (ws_bytes < embedding_bytes(tokens, cols)) return SRQ_ERR_WORKSPACE;
    if (empty(rows, cols) || (accumulate && tokens == 0)) return SRQ_OK;
    const EmbedBwdArgs a = {dout, dt, tokens, cols, ld, ids, id_t, rows, scale, dtable, dtable_dt, ld_dtable, accumulate, ws, device_status};
    return status_of(launch_embedding_bwd(a, (cudaStream_t)cuda_stream));
}

srq_status_t srq_logprob_fwd(const void* logits, srq_dtype_t dt, int64_t rows, int64_t classes, int64_t ld, const void* targets, srq_index_t target_t,
                             float temperature, float* logp, float* lse, uint32_t* device_status, void* cuda_stream) {
    SRQ_TRY(check_logits(logits, dt, rows, classes, ld, targets, target_t, temperature, device_status));
    if ((!logp && rows) || !aligned_to(logp, 4) || !aligned_to(lse, 4)) return SRQ_ERR_INVALID_ARG;
    if (rows == 0) return SRQ_OK;
    const LogitsArgs a = {logits, dt, rows, classes, ld, targets, target_t, temperature, device_status};
    return status_of(launch_logprob_fwd(a, logp, lse, (cudaStream_t)cuda_stream));
}

srq_status_t srq_logprob_bwd(const void* logits, srq_dtype_t dt, int64_t rows, int64_t classes, int64_t ld, const void* targets, srq_index_t target_t,
                             float temperature, const float* lse, const float* dlogp, void* dlogits, int64_t ld_dlogits, uint32_t* device_status,
                             void* cuda_stream) {
    SRQ_TRY(check_logits(logits, dt, rows, classes, ld, targets, target_t, temperature, device_status));
    if ((!lse && rows) || (!dlogp && rows) || !aligned_to(lse, 4) || !aligned_to(dlogp, 4)) return SRQ_ERR_INVALID_ARG;
    if (!dlogits && !empty(rows, classes)) return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_dlogits(logits, ld, dlogits, ld_dlogits, classes));
    if (empty(rows, classes)) return SRQ_OK;
    const LogitsArgs a = {logits, dt, rows, classes, ld, targets, target_t, temperature, device_status};
    return status_of(launch_logprob_bwd(a, lse, dlogp, dlogits, ld_dlogits, (cudaStream_t)cuda_stream));
}

srq_status_t srq_policy_loss(const void* logits, srq_dtype_t dt, int64_t rows, int64_t classes, int64_t ld, const void* targets, srq_index_t target_t,
                             const float* logp_old, const float* advantage, const float* weight, const float* logp_ref, const srq_policy_t* policy,
                             float* row_loss, float* loss, float* logp, void* dlogits, int64_t ld_dlogits, uint32_t* device_status, void* cuda_stream) {
    if (!policy) return SRQ_ERR_INVALID_ARG;
    const srq_policy_t& h = *policy;
    SRQ_TRY(check_logits(logits, dt, rows, classes, ld, targets, target_t, h.temperature, device_status));
    if (!(h.clip_low >= 0.0f) || !(h.clip_high >= 0.0f) || !(h.kl_coef >= 0.0f) || !isfinite(h.kl_coef)) return SRQ_ERR_INVALID_ARG;
    if (rows && (!logp_old || !advantage || !weight)) return SRQ_ERR_INVALID_ARG;
    if (!row_loss && !logp && !dlogits && !empty(rows, classes)) return SRQ_ERR_INVALID_ARG;
    if (loss && !row_loss && rows) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(logp_old, 4) || !aligned_to(advantage, 4) || !aligned_to(weight, 4) || !aligned_to(logp_ref, 4) || !aligned_to(row_loss, 4) ||
        !aligned_to(loss, 4) || !aligned_to(logp, 4))
        return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_dlogits(logits, ld, dlogits, ld_dlogits, classes));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) return loss ? status_of(cudaMemsetAsync(loss, 0, 4, st)) : SRQ_OK;
    const LogitsArgs a = {logits, dt, rows, classes, ld, targets, target_t, h.temperature, device_status};
    const PolicyArgs p = {logp_old, advantage, weight, logp_ref, h, row_loss, loss, logp, dlogits, ld_dlogits};
    return status_of(launch_policy(a, p, st));
}

size_t srq_preference_workspace_bytes(int64_t rows) {
    if (rows < 0 || rows > kMaxExtent) return 0;
    return align_up(preference_bytes(rows) + 1);
}

srq_status_t srq_preference_loss(const void* logits, srq_dtype_t dt, int64_t rows, int64_t classes, int64_t ld, const void* targets, srq_index_t target_t,
                                 const float* logp_ref, const void* offsets, srq_index_t offset_t, int64_t pairs, const srq_preference_t* preference,
                                 float* pair_loss, float* loss, float* logp, void* dlogits, int64_t ld_dlogits, void* ws, size_t ws_bytes,
                                 uint32_t* device_status, void* cuda_stream) {
    if (!preference) return SRQ_ERR_INVALID_ARG;
    const srq_preference_t& h = *preference;
    SRQ_TRY(check_logits(logits, dt, rows, classes, ld, targets, target_t, h.temperature, device_status));
    if (!isfinite(h.beta) || !(h.label_smoothing >= 0.0f && h.label_smoothing <= 1.0f) || pairs < 0 || !known_index(offset_t)) return SRQ_ERR_INVALID_ARG;
    if (h.clear_rest != 0 && h.clear_rest != 1) return SRQ_ERR_INVALID_ARG;
    if (pairs > kMaxExtent / 2) return SRQ_ERR_UNSUPPORTED;
    if ((rows && (!logp_ref || !logp)) || (pairs && (!pair_loss || !offsets))) return SRQ_ERR_INVALID_ARG;
    if (!aligned_to(logp_ref, 4) || !aligned_to(offsets, index_bytes(offset_t)) || !aligned_to(pair_loss, 4) || !aligned_to(loss, 4) || !aligned_to(logp, 4))
        return SRQ_ERR_INVALID_ARG;
    SRQ_TRY(check_dlogits(logits, ld, dlogits, ld_dlogits, classes));
    if (!ws || !aligned_to(ws, 256)) return SRQ_ERR_INVALID_ARG;
    if (ws_bytes < srq_preference_workspace_bytes(rows)) return SRQ_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (pairs == 0) {                                          // no row belongs to an answer
        const size_t esize = dt == SRQ_F32 ? 4 : 2;
        if (h.clear_rest && rows) SRQ_TRY(status_of(cudaMemsetAsync(logp, 0, (size_t)rows * 4, st)));
        if (h.clear_rest && dlogits && !empty(rows, classes))
            SRQ_TRY(status_of(cudaMemset2DAsync(dlogits, (size_t)ld_dlogits * esize, 0, (size_t)classes * esize, (size_t)rows, st)));
        return loss ? status_of(cudaMemsetAsync(loss, 0, 4, st)) : SRQ_OK;
    }
    const LogitsArgs a = {logits, dt, rows, classes, ld, targets, target_t, h.temperature, device_status};
    const PreferenceArgs p = {logp_ref, offsets, offset_t, pairs, h, pair_loss, loss, logp, dlogits, ld_dlogits};
    return status_of(launch_preference(a, p, ws, st));
}

srq_status_t srq_adamw_step(const srq_adamw_tensor_t* tensors, int64_t count, srq_dtype_t param_dt, srq_dtype_t grad_dt, int32_t state_bits,
                            const srq_adamw_t* adamw, uint32_t* device_status, void* cuda_stream) {
    if (count < 0 || (count && !tensors) || !adamw || !known_dtype(param_dt) || !known_dtype(grad_dt)) return SRQ_ERR_INVALID_ARG;
    if (state_bits != 8 && state_bits != 32) return SRQ_ERR_UNSUPPORTED;
    const srq_adamw_t& h = *adamw;
    if (!isfinite((float)h.lr) || !isfinite((float)h.weight_decay) || !(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0)) return SRQ_ERR_INVALID_ARG;
    if (!((float)h.eps >= 0x1p-126f) || !isfinite((float)h.eps) || h.step < 1) return SRQ_ERR_INVALID_ARG;
    if (h.round != SRQ_SR && h.round != SRQ_RTN && h.round != SRQ_SR8 && h.round != SRQ_RNE) return SRQ_ERR_INVALID_ARG;
    if (h.round != SRQ_SR && h.round != SRQ_RNE) return SRQ_ERR_UNSUPPORTED;
    if (!aligned_to(h.lr_device, 4) || !aligned_to(h.step_device, 8) || !aligned_to(h.grad_scale, 4) || !aligned_to(device_status, 4)) return SRQ_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        const srq_adamw_tensor_t& t = tensors[i];
        if (t.n < 0) return SRQ_ERR_INVALID_ARG;
        if (t.n && (!t.param || !t.grad || !t.m || !t.v)) return SRQ_ERR_INVALID_ARG;
        if (!aligned_to(t.param, 16) || !aligned_to(t.grad, 16) || !aligned_to(t.m, 16) || !aligned_to(t.v, 16)) return SRQ_ERR_INVALID_ARG;
        if (state_bits == 8 && ((t.n && (!t.m_step || !t.v_step)) || !aligned_to(t.m_step, 4) || !aligned_to(t.v_step, 4))) return SRQ_ERR_INVALID_ARG;
    }
    if (count == 0) return SRQ_OK;
    const AdamwArgs a = {tensors, count, param_dt, grad_dt, state_bits == 8, h.round == SRQ_SR, adamw, device_status};
    return status_of(launch_adamw(a, (cudaStream_t)cuda_stream));
}

}  // extern "C"
