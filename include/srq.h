/*
 * srq — stochastically-rounded quantized linear layer for NVIDIA B200 (sm_100a).
 *
 * C ABI of libsrq.so.  The operations are those of the paper "Training with
 * Fewer Bits: Unlocking Edge LLMs Training with Stochastic Rounding":
 * the threshold quantizer Q_D(x, eps) (Def. 1) in its round-to-nearest
 * (Def. 2) and stochastic-rounding (Def. 3) forms, the mixed-precision
 * forward pass (Alg. 1) and the mixed-precision backward pass (Alg. 2).
 *
 * Conventions for every entry point
 *   - Storage: activations A[T,K], weights W[N,K], output gradients dY[T,N],
 *     all row-major; Y[T,N] = Q(A) Q(W)^T, dA[T,K] = Q(dY) Q(W),
 *     dW[N,K] = Q(dY)^T Q(A).  (The paper writes W as [in,out]; this is the
 *     same mathematics with W stored [out,in].)
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, the
 *     workspace included.  qspec pointers and the debug struct are HOST
 *     pointers, read before the call returns.  The library allocates no
 *     device memory.  Between calls it keeps only what it has learned about the
 *     devices (SM count, how many CTAs of a kernel fit, the address of the array
 *     sr_quantize_static uses; each found once, thread-safely) and the launch
 *     counter of srq_launch_count; nothing of it changes a result.
 *     (sr_quantize_static is the one exception to "no device memory": see there.)
 *   - Work is enqueued on `cuda_stream` (a cudaStream_t passed as void*, NULL
 *     for the default stream) and the call returns without waiting.
 *   - Errors the host can see (null pointer, bits outside the grid's range, a pitch or
 *     pointer that breaks the alignment rules below, workspace too small,
 *     a contraction long enough to overflow int32) return a status at once
 *     and enqueue nothing.  Conditions only the device can see (an input
 *     that is not finite, a bounded wait inside a kernel that ran out) are
 *     recorded in a status word at the start of the workspace; read it with
 *     srq_poll_status (sr_quantize_static, which has no workspace, reports
 *     through a word the caller passes).  After such a condition the outputs are
 *     unspecified.
 *   - Outputs are overwritten, unless a srq_output_t (the *_ex entry points) asks for accumulation.
 *   - Both operands of a layer pass use the same grid (srq_qspec_t.format).  With the
 *     floating-point grid (E4M3, or E4M2 / E4M1 / E4M0 by `bits`) the codes are E4M3 bytes,
 *     D_g = absmax_g / (largest value of the grid: 448, 448, 384, 256), the products run in
 *     kind::f8f6f4 with binary32 accumulation, and the `acc` member of the debug struct receives
 *     binary32 sums (same size as int32).
 *   - Alignment: input base pointers 16-byte aligned; input pitch `ld` in
 *     elements; fp32 outputs 16-byte aligned; the workspace 256-byte aligned.
 *     Inputs whose pitch or extent is not a multiple of 4 elements take a
 *     slower element-wise path with identical results.
 *
 * Step size.  The paper leaves the precision level D of Def. 1 free.  Here
 * D_g = absmax_g / qmax with qmax = 2^(bits-1) - 1 and codes in
 * [-qmax, qmax]; x / D is evaluated as x * inv_g, one binary32 multiply,
 * with inv_g = qmax / absmax_g rounded toward zero, so that the quotient of
 * every element of the group stays within [-qmax, qmax] as in Def. 1.  The group g is the whole tensor (SRQ_PER_TENSOR) or one row of
 * the code layout being written (SRQ_PER_ROW), i.e. one index of the
 * dimension that is NOT contracted in the product that consumes the codes.
 *
 * Thresholds.  eps of Def. 3 is never stored: element x[r,c] uses
 * eps = u24 * 2^-24, where u24 is the top 24 bits of word (i & 3) of
 * Philox4x32-10 with counter {lo(i>>2), hi(i>>2), lo(tensor_id),
 * hi(tensor_id)} and key {lo(seed), hi(seed)}, i = index_offset + r*cols + c.
 * SR rounds up iff eps < frac(x/D); RTN rounds up iff frac(x/D) >= 1/2.
 * The same (seed, tensor_id, index_offset, bits, scale, round) reproduces the
 * same codes, which is how one quantized W serves forward and backward.
 */
#ifndef SRQ_H
#define SRQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SRQ_OK = 0,
    SRQ_ERR_INVALID_ARG = 1,   /* null pointer, bad enum, bad extent, misaligned pointer/pitch */
    SRQ_ERR_UNSUPPORTED = 2,   /* bits outside 2..8 (5..8 on the floating-point grid); options that do not combine */
    SRQ_ERR_WORKSPACE = 3,     /* workspace smaller than srq_*_workspace_bytes says */
    SRQ_ERR_ACC_OVERFLOW = 4,  /* contraction length * qmax_a * qmax_b >= 2^31 */
    SRQ_ERR_CUDA = 5,          /* a CUDA call failed (launch, tensor-map encode, copy) */
    SRQ_ERR_NONFINITE = 6,     /* device: an input group has a NaN or infinite absmax */
    SRQ_ERR_TIMEOUT = 7        /* device: a bounded wait in a kernel ran out */
} srq_status_t;

typedef enum { SRQ_F32 = 0, SRQ_BF16 = 1 } srq_dtype_t;
/* SRQ_PER_BLOCK: one step size per block of 128 values; the srq_*_blocks and srq_rmsnorm / srq_glu entry points
 * only (the block's shape is srq_blocks_t.tile_rows), which take no other mode. */
typedef enum { SRQ_PER_TENSOR = 0, SRQ_PER_ROW = 1, SRQ_PER_BLOCK = 2 } srq_scale_t;
/* SRQ_SR8: stochastic rounding with 8 random bits per element instead of 24 (the paper's hardware
 * section argues that a few pseudo-random bits per rounding suffice): eps = (b + 1/2) / 256 with b
 * byte (i & 3) of word ((i >> 2) & 3) of Philox block i >> 4, so that one block serves 16 elements.
 * P(round up) is the fraction rounded to the nearest 1/256.  Integer grid only. */
typedef enum { SRQ_SR = 0, SRQ_RTN = 1, SRQ_SR8 = 2, SRQ_RNE = 3 /* nearest, ties to even; block entry points only */ } srq_round_t;
/* Grid of a quantization point: integers times the step size (bits 2..8), or 8-bit floating-point
 * values times the step size.  SRQ_GRID_E4M3 with bits = 8 is E4M3 (1 sign, 4 exponent, 3 mantissa
 * bits, bias 7, no infinities, largest value 448); bits = 7, 6, 5 select E4M2, E4M1, E4M0, the
 * formats of the paper's experiments section, taken as the E4M3 values with 2, 1, 0 mantissa bits
 * (largest values 448, 384, 256; Def. 1 with the binade's own step).  Their codes are E4M3 bytes
 * with the low mantissa bits clear, so one product (kind::f8f6f4) serves all four. */
typedef enum { SRQ_GRID_INT = 0, SRQ_GRID_E4M3 = 1, SRQ_GRID_NONE = 2 /* operand left unquantized */ } srq_grid_t;

/* One quantization point: the paper's (D, eps) pair for one operand of one pass
 * (five per layer: A and W forward; A, W and dY backward). */
typedef struct {
    int32_t bits;          /* integer grid: 2..8 (codes are stored one per int8 whatever the width);
                              floating-point grid: 8, 7, 6, 5 = E4M3, E4M2, E4M1, E4M0 */
    int32_t scale;         /* srq_scale_t */
    int32_t round;         /* srq_round_t */
    int32_t format;        /* srq_grid_t; 0 = integer grid */
    uint64_t seed;         /* Philox key; one per training step */
    uint64_t tensor_id;    /* Philox counter words 2-3; one per (layer, operand, pass) */
    uint64_t index_offset; /* added to the flat index; first_row*cols for a row shard */
    const float *absmax;   /* optional, DEVICE pointer.  SRQ_PER_TENSOR: one float, max |x| of the operand
                            * when the caller already knows it (srq_absmax, or an all-reduced maximum
                            * over token shards); the absmax pass over the operand is then skipped.
                            * SRQ_PER_ROW: [cols] floats, max |x[:, c]| of every column of the source
                            * matrix (srq_absmax_cols, max-reduced over token shards), used for the
                            * step sizes of the TRANSPOSED layout, whose groups run over the rows,
                            * i.e. over tokens other shards may hold; the row-major layout's row
                            * maxima are always computed here.  Values must not be smaller than the
                            * true maxima (codes are unspecified otherwise).  NULL: compute them. */
} srq_qspec_t;

/* Optional copies of what a layer pass fed to its product: dense code matrices in the layout
 * the product consumed (contracted axis contiguous), their step sizes, and the int32 sums.
 * Any member may be NULL.  All are device pointers. */
typedef struct {
    int8_t *codes_a;   /* first operand  [M, Kc] */
    float *scale_a;    /* [1] or [M] */
    int8_t *codes_b;   /* second operand [Nn, Kc] */
    float *scale_b;    /* [1] or [Nn] */
    int32_t *acc;      /* [M, Nn] */
} srq_debug_out_t;

/* Bytes of workspace sr_quantize needs for a [rows, cols] input. */
size_t srq_quantize_workspace_bytes(int64_t rows, int64_t cols);

/* Bytes of workspace srq_gemm_i8 needs for an [M, N] output (partial sums of a split contraction). */
size_t srq_gemm_workspace_bytes(int64_t M, int64_t N);

/* Bytes of workspace that suffices for any one of the qlinear_* calls on a layer with
 * T tokens, N output and K input features. */
size_t srq_workspace_bytes(int64_t T, int64_t N, int64_t K);

/*
 * Def. 1-3 applied element-wise to x[rows, cols] (row pitch ld elements, type dt).
 * Writes int8 codes in the row-major layout codes_rm[rows, ld_rm] with scale_rm ([1] per
 * tensor, [rows] per row) and/or the transposed layout codes_tr[cols, ld_tr] with scale_tr
 * ([1] per tensor, [cols] per row of that layout, i.e. per column of x).  A NULL code
 * pointer skips that layout (its scale pointer is then ignored).  Per tensor both layouts
 * hold the same codes; per row they differ in step size but share each element's threshold.
 * ld_rm >= cols, ld_tr >= rows; padding bytes are left untouched.
 */
srq_status_t sr_quantize(const void *x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld,
                         const srq_qspec_t *q,
                         int8_t *codes_rm, int64_t ld_rm, float *scale_rm,
                         int8_t *codes_tr, int64_t ld_tr, float *scale_tr,
                         void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * sr_quantize for callers that cannot allocate device memory.  (The paper has no counterpart
 * of this entry point; it exists for deployment reasons only.)  Same operation, arguments and
 * results as sr_quantize, but without a workspace: the scratch words come from a 1 MiB array
 * built into the library, which every device that loads the library holds until the process
 * exits.  Meant for code that runs where cudaMalloc is unavailable or unwelcome: inside a
 * framework whose memory pool is already fully assigned, in a plug-in that is handed only its
 * input and output tensors, or in a latency-critical loop that must not hit the allocator's
 * implicit synchronisation.  The call itself allocates nothing, on the host or the device.
 *   - Limit: 512 + 2 * (pad64(rows) + pad64(cols)) * 4 bytes must fit in 1 MiB, pad64 rounding
 *     up to a multiple of 64 (about rows + cols <= 131000); larger inputs return
 *     SRQ_ERR_WORKSPACE and enqueue nothing.
 *   - The first call on each device looks up the array's device address (with that device
 *     current).  Make that first call outside any stream capture.
 *   - device_status: optional caller-owned device word (4-byte aligned) that is cleared and
 *     then receives SRQ_ERR_NONFINITE if an input group is not finite; pass NULL to ignore.
 *   - All calls on a device share the array, and it keeps the previous call's contents; each
 *     call clears what it needs.  Calls whose kernels may overlap on the same device (streams
 *     with no ordering between them) race with each other: order them, or use sr_quantize.
 */
srq_status_t sr_quantize_static(const void *x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld,
                                const srq_qspec_t *q,
                                int8_t *codes_rm, int64_t ld_rm, float *scale_rm,
                                int8_t *codes_tr, int64_t ld_tr, float *scale_tr,
                                uint32_t *device_status, void *cuda_stream);

/* max |x| over x[rows, cols] (row pitch ld elements) into *absmax (device, one float), e.g. to
 * share it between the forward and the backward quantization point of the same tensor, or to
 * all-reduce it over token shards, through srq_qspec_t.absmax.  Needs no workspace. */
srq_status_t srq_absmax(const void *x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld,
                        float *absmax, void *cuda_stream);

/* max |x[:, c]| of every column into absmax_cols (device, [cols] floats, overwritten): what a token
 * shard contributes to the per-row step sizes of the transposed layout (the operands of the
 * weight-gradient product); max-reduce it over the shards and pass it through srq_qspec_t.absmax. */
srq_status_t srq_absmax_cols(const void *x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld,
                             float *absmax_cols, void *cuda_stream);

/*
 * The product of two quantized matrices (mixed-precision matmul subsection): int8 codes
 * a[M, Kc] (pitch lda) and b[N, Kc] (pitch ldb), both with the contracted axis contiguous,
 * multiplied on the tensor cores with exact int32 accumulation, then
 *     out[i, j] = float(acc[i, j]) * (s_row[i * row_stride] * s_col[j * col_stride])
 * (each operation one binary32 rounding).  row_stride / col_stride are 0 for a per-tensor
 * step size and 1 for per-row.  acc_out, if not NULL, also receives the raw sums [M, N]
 * (pitch N).  lda and ldb must be multiples of 16 and a, b 16-byte aligned (TMA rule).
 * Requires Kc * 127 * 127 < 2^31 unless the caller passes smaller code ranges through the
 * qlinear_* entry points, which check the bound for their own bit widths.
 */
srq_status_t srq_gemm_i8(const int8_t *a, int64_t lda, const int8_t *b, int64_t ldb,
                         int64_t M, int64_t N, int64_t Kc,
                         const float *s_row, int32_t row_stride,
                         const float *s_col, int32_t col_stride,
                         float *out, int64_t ldo, int32_t *acc_out,
                         void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The same product for E4M3 codes (the 8-bit floating-point grid; the paper's experiments use
 * the E4M0 / E4M1 / E4M2 members of this family): a[M, Kc], b[N, Kc] are E4M3 bytes, multiplied
 * on the tensor cores (kind::f8f6f4) with binary32 accumulation, whose summation order is the
 * hardware's, so results agree with the exact product to about 1e-5 * |row| * |col| rather than
 * bit for bit.  out[i, j] = acc[i, j] * (s_row[i] * s_col[j]); acc_out, if not NULL, receives
 * the raw binary32 sums [M, N].  Alignment rules as for srq_gemm_i8; the contraction is never
 * split, so the workspace only needs its 256-byte header.
 */
srq_status_t srq_gemm_e4m3(const uint8_t *a, int64_t lda, const uint8_t *b, int64_t ldb,
                           int64_t M, int64_t N, int64_t Kc,
                           const float *s_row, int32_t row_stride,
                           const float *s_col, int32_t col_stride,
                           float *out, int64_t ldo, float *acc_out,
                           void *ws, size_t ws_bytes, void *cuda_stream);

/* Alg. 1: Y[T,N] = Q(A) Q(W)^T.  qA, qW are the forward quantization points of A and W.
 * Per row: A per token, W per output feature.
 * qA->format == SRQ_GRID_NONE gives the forward pass of the paper's mixed-precision SGD for the
 * quantization-aware objective, which leaves the forward activations unquantized (D_A^fwd = 0):
 * Y = A Q(W)^T with A used as the bfloat16 numbers it holds (dt must be SRQ_BF16, K a multiple
 * of 8, W on the integer grid).  The product then runs in bfloat16 with binary32 accumulation,
 * so Y agrees with the exact product to about 1e-5 * |row| * |col| rather than bit for bit; dbg
 * is ignored. */
srq_status_t qlinear_fwd(const void *A, const void *W, srq_dtype_t dt,
                         int64_t T, int64_t N, int64_t K,
                         const srq_qspec_t *qA, const srq_qspec_t *qW,
                         float *Y, const srq_debug_out_t *dbg,
                         void *ws, size_t ws_bytes, void *cuda_stream);

/* Alg. 2, input gradient: dA[T,K] = Q(dY) Q(W).  The contraction runs over N, so Q(W) is
 * written in its transposed layout [K,N].  Per row: dY per token, W per input feature. */
srq_status_t qlinear_bwd_input(const void *dY, const void *W, srq_dtype_t dt,
                               int64_t T, int64_t N, int64_t K,
                               const srq_qspec_t *qdY, const srq_qspec_t *qW,
                               float *dA, const srq_debug_out_t *dbg,
                               void *ws, size_t ws_bytes, void *cuda_stream);

/* Alg. 2, weight gradient: dW[N,K] = Q(dY)^T Q(A).  The contraction runs over the T tokens;
 * both operands are written in their transposed layouts [N,T] and [K,T].  Per row: dY per
 * output feature, A per input feature. */
srq_status_t qlinear_bwd_weight(const void *dY, const void *A, srq_dtype_t dt,
                                int64_t T, int64_t N, int64_t K,
                                const srq_qspec_t *qdY, const srq_qspec_t *qA,
                                float *dW, const srq_debug_out_t *dbg,
                                void *ws, size_t ws_bytes, void *cuda_stream);

/* Alg. 2 as a whole: dA[T,K] = Q(dY) Q(W) and dW[N,K] = Q(dY)^T Q(A) in one call.  Alg. 2
 * quantizes dY once and uses it in both products; here dY is read once and its codes are written
 * in both layouts ([T,N] for dA, [N,T] for dW) by the same pass, which saves one absmax and one
 * quantization pass over dY compared with qlinear_bwd_input followed by qlinear_bwd_weight.  The
 * results are bit for bit those of the two separate calls with the same quantization points.
 * dbg_input / dbg_weight receive the operands and sums of the dA and dW products. */
srq_status_t qlinear_bwd(const void *dY, const void *A, const void *W, srq_dtype_t dt,
                         int64_t T, int64_t N, int64_t K,
                         const srq_qspec_t *qdY, const srq_qspec_t *qA, const srq_qspec_t *qW,
                         float *dA, float *dW,
                         const srq_debug_out_t *dbg_input, const srq_debug_out_t *dbg_weight,
                         void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * What else a product does with its results; every member is optional (zero / NULL).
 *   accumulate  1: out += result (one binary32 addition per element) instead of out = result.
 *               The paper emulates large batches by accumulating gradients over micro-batches
 *               (hardware-considerations section); this is that accumulation for dW.
 *               2: the int32 sums are accumulated instead: acc_out += sums (the call's acc_out /
 *               dbg->acc matrix is required and holds the running sums; zero it before the first
 *               micro-batch) and out = float(acc_out) * (s_row * s_col) is written from the total.
 *               Exact - the result equals one product over the concatenated contraction - as
 *               long as every micro-batch uses the same step sizes (srq_qspec_t.absmax) and the
 *               totals fit int32; a wrap is reported as SRQ_ERR_ACC_OVERFLOW by srq_poll_status.
 *               Integer grid only.
 *   q, step, codes, ld_codes
 *               also write Q(result) as int8 codes [M, ld_codes] for the layer that consumes the
 *               result (the next layer's Q(A_in) of Alg. 1, the previous layer's Q(dA_out) of
 *               Alg. 2), fused into the product's epilogue so that the result is not read again.
 *               The absmax of a result is not known until the product has finished, so the step
 *               size comes from the caller: *step (device, [1]); x / D is out * (1 / D) with one
 *               binary32 division, SATURATED to [-qmax, qmax], then rounded by q->round with the
 *               thresholds of (q->seed, q->tensor_id, q->index_offset + i * N + j).  q must be on
 *               the integer grid; q->scale is ignored (one step for the whole result).  With
 *               codes given, the fp32 output pointer of the call may be NULL.
 *   absmax      device [1], holding a non-negative number (usually 0) on entry: raised to
 *               max |result|, from which the caller derives the step size of its next step.
 *   out_bf16    1: the output pointer of the call addresses bfloat16 numbers (pass it cast to
 *               float *; its pitch counts bfloat16 elements): each binary32 result is rounded to
 *               the nearest bfloat16, ties to even, as it is stored, which halves the bytes the
 *               product writes.  Codes and absmax still come from the binary32 result.  Not with
 *               accumulate = 1 (SRQ_ERR_UNSUPPORTED): running binary32 sums stay in binary32.
 *   raw_sums    1: the output pointer of the call addresses int32 numbers (pass it cast to float *;
 *               its pitch counts int32 elements) and receives the exact sums themselves; nothing
 *               is scaled.  For token shards on several devices (the batch axis of the variance
 *               lemma): the shards' sums are added with an integer all-reduce, which is exact in
 *               any order, and srq_dequant_i32 then scales the total once, so that the weight
 *               gradient is bit for bit the one a single device computes on the whole batch
 *               (given shared step sizes, srq_qspec_t.absmax).  Integer grid only; not combined
 *               with any other member (SRQ_ERR_UNSUPPORTED).
 * Products with q or absmax set are never split along the contraction.
 */
typedef struct {
    int32_t accumulate;
    int32_t out_bf16;
    const srq_qspec_t *q;
    const float *step;
    int8_t *codes;
    int64_t ld_codes;
    float *absmax;
    int32_t raw_sums;
} srq_output_t;

/* srq_gemm_i8, qlinear_fwd and qlinear_bwd with output options (NULL = none, i.e. the plain call).
 * In qlinear_bwd_ex, output_dA applies to dA[T,K] and output_dW to dW[N,K]. */
srq_status_t srq_gemm_i8_ex(const int8_t *a, int64_t lda, const int8_t *b, int64_t ldb,
                            int64_t M, int64_t N, int64_t Kc,
                            const float *s_row, int32_t row_stride,
                            const float *s_col, int32_t col_stride,
                            float *out, int64_t ldo, int32_t *acc_out, const srq_output_t *output,
                            void *ws, size_t ws_bytes, void *cuda_stream);
srq_status_t qlinear_fwd_ex(const void *A, const void *W, srq_dtype_t dt,
                            int64_t T, int64_t N, int64_t K,
                            const srq_qspec_t *qA, const srq_qspec_t *qW, float *Y,
                            const srq_output_t *output, const srq_debug_out_t *dbg,
                            void *ws, size_t ws_bytes, void *cuda_stream);
srq_status_t qlinear_bwd_ex(const void *dY, const void *A, const void *W, srq_dtype_t dt,
                            int64_t T, int64_t N, int64_t K,
                            const srq_qspec_t *qdY, const srq_qspec_t *qA, const srq_qspec_t *qW,
                            float *dA, float *dW,
                            const srq_output_t *output_dA, const srq_output_t *output_dW,
                            const srq_debug_out_t *dbg_input, const srq_debug_out_t *dbg_weight,
                            void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The finishing step of a product on its own (the last line of Alg. 1 / Alg. 2 once the integer
 * sums exist): out[i, j] = float(acc[i, j]) * (s_row[i * row_stride] * s_col[j * col_stride]) over a
 * caller's int32 matrix acc[M, N] (pitch ld_acc), with the same three roundings in the same order as
 * the products' own epilogue, so that sums collected with raw_sums and scaled here give the very
 * bits the one-call product gives.  out is binary32 [M, ldo], or bfloat16 when out_bf16 = 1 (round
 * to nearest even).  All pointers are device pointers, 4-byte aligned (16-byte alignment and
 * pitches that are multiples of 4 allow vector accesses).  Needs no workspace.
 */
srq_status_t srq_dequant_i32(const int32_t *acc, int64_t ld_acc, int64_t M, int64_t N,
                             const float *s_row, int32_t row_stride,
                             const float *s_col, int32_t col_stride,
                             void *out, int64_t ldo, int32_t out_bf16, void *cuda_stream);

/* ------------------------------------------------------------------------------------------------
 * Block-scaled E4M3 operators: the quantizer, the product, the norm and the gated feed-forward block around
 * a linear layer, with one step size for every 128 values along the contracted axis (1 x 128) or for every
 * 128 x 128 tile.  Finer step sizes keep a few large activations from costing all the others their precision;
 * the products take the step sizes apart again: every 128-long piece of the contraction is summed on the
 * tensor cores in binary32 and scaled before it is added to the total.
 *
 * Conventions, where they differ from the calls above
 *   - No workspace and no header: `device_status` is an optional caller-owned device word (4-byte aligned).
 *     A call does not clear it; it receives SRQ_ERR_NONFINITE or SRQ_ERR_TIMEOUT if the device meets such a
 *     condition and it holds zero.  Zero it once, read it after as many calls as you like.  Values that are not
 *     finite are looked for where step sizes are formed (every block that is coded) and in the norm's forward pass,
 *     which also reports rows of finite values whose mean square is not finite in binary32 (or zero with eps = 0);
 *     what leaves in 16 or 32 bits only is not searched.
 *   - Step size of a block: D = absmax / 448, the quotient is x * inv with inv = 448 / absmax rounded toward
 *     zero; a block whose absmax is 0 or at most 7 * 2^-122 (the reciprocal would overflow) has D = 0 and
 *     codes 0.
 *   - Rounding: SRQ_RNE (nearest, ties to even, the conversion instruction's rule) or SRQ_SR (Def. 3, with the
 *     thresholds of the flat index in the matrix that is being quantized, the source's own for both
 *     layouts).  q->bits must be 8, q->format SRQ_GRID_E4M3, q->scale SRQ_PER_BLOCK; q->absmax is ignored.
 *   - The last block of a row may be shorter than 128.
 *   - Extents may be 0.  An operand without elements may have null pointers, and a call whose result has none does
 *     nothing; sums over nothing (Kc = 0, a weight's gradient over no rows) are written as zero.  srq_glu_fwd wants
 *     K >= 1.
 */

/* A matrix of E4M3 codes [rows, cols] with its step sizes, on the device: element (r, c) stands for
 * code * scale[(r / tile_rows) * ld_scale + c / 128]. */
typedef struct {
    uint8_t *codes;      /* [rows, ld], 16-byte aligned; padding bytes are neither read nor written */
    int64_t ld;          /* pitch in bytes, >= cols, a multiple of 16 */
    float *scale;        /* [ceil(rows / tile_rows), ld_scale], 4-byte aligned */
    int64_t ld_scale;    /* pitch in floats, >= ceil(cols / 128); a multiple of 4 with a 16-byte aligned base is faster */
    int32_t tile_rows;   /* 1: blocks of 1 x 128; 128: tiles of 128 x 128 */
} srq_blocks_t;

/* x[rows, cols] (pitch ld elements; 16-byte aligned base) as block codes: row-major into rm (blocks along the
 * columns of x) and / or transposed into tr (a [cols, rows] matrix, blocks along the rows of x); NULL skips a
 * layout.  With tile_rows = 128 both layouts hold the same codes and step sizes (transposed). */
srq_status_t srq_quantize_blocks(const void *x, srq_dtype_t dt, int64_t rows, int64_t cols, int64_t ld,
                                 const srq_qspec_t *q, const srq_blocks_t *rm, const srq_blocks_t *tr,
                                 uint32_t *device_status, void *cuda_stream);

/* The same for a source that is itself block-coded (an 8-bit activation checkpoint): its numbers are
 * formed in binary32 and quantized anew, e.g. turned over for a contraction over the tokens. */
srq_status_t srq_requantize_blocks(const srq_blocks_t *x, int64_t rows, int64_t cols,
                                   const srq_qspec_t *q, const srq_blocks_t *rm, const srq_blocks_t *tr,
                                   uint32_t *device_status, void *cuda_stream);

/* out[M, N] (+)= A B^T, A[M, Kc] and B[N, Kc] block-coded with the contracted axis contiguous:
 *   out[i, j] = sum over blocks k of  sA[i, k] * sB[j, k] * sum_{c in block k} a[i, c] * b[j, c]
 * in binary32, the inner sums on the tensor cores; sA * sB is formed first, so that it has to stay within binary32's
 * normal range for a result of full precision.  out is binary32 or bfloat16 (out_dt, rounded once, to
 * nearest even), pitch ldo elements.  accumulate = 1 adds to a binary32 out instead of overwriting it.  Any M
 * from one token up; the sum's order depends on sizes, types, alignment and the device alone, so that the same
 * call repeats bit for bit (with accumulate = 1 too: one addition per element). */
srq_status_t srq_gemm_blocks(const srq_blocks_t *a, const srq_blocks_t *b, int64_t M, int64_t N, int64_t Kc,
                             void *out, srq_dtype_t out_dt, int64_t ldo, int32_t accumulate,
                             uint32_t *device_status, void *cuda_stream);

/* Root-mean-square norm with the residual's addition, output as block codes (tile_rows = 1):
 *   r = x + residual (residual may be NULL: r = x),  rstd = 1 / sqrt(mean(r^2) + eps),  y = r * rstd * w.
 * x, residual and r_out have type dt and pitches in elements, w[cols] type w_dt; everything is computed in
 * binary32 from the unrounded sum r.  y (block codes of y), y_out (y itself, type dt), r_out (r, rounded to
 * dt) and rstd ([rows], for the backward pass) may each be NULL, but not y and y_out both.
 * Base pointers are 16-byte aligned; pitches that are multiples of 8 elements and extents that are multiples
 * of 8 take the vector path. */
srq_status_t srq_rmsnorm_fwd(const void *x, int64_t ldx, const void *residual, int64_t ld_residual, srq_dtype_t dt,
                             const void *w, srq_dtype_t w_dt, int64_t rows, int64_t cols, float eps,
                             const srq_qspec_t *q, const srq_blocks_t *y, void *y_out, int64_t ld_y,
                             void *r_out, int64_t ld_r, float *rstd, uint32_t *device_status, void *cuda_stream);

/* Bytes of workspace srq_rmsnorm_bwd needs when dw is wanted (at most 512 partial rows of the weight's gradient). */
size_t srq_rmsnorm_workspace_bytes(int64_t rows, int64_t cols);

/* Its backward pass.  With n = r * rstd:
 *   dx = rstd * (w * dy - n * mean(w * dy * n)) + d_residual      (the gradient of x and of the residual)
 *   dw = sum over rows of dy * n                                    (binary32 [cols])
 * dy is the gradient at y, d_residual (optional) the one that arrives at r, r is srq_rmsnorm_fwd's r_out (x
 * where it had no residual).  dx or dw may be NULL.  The sum over rows has a fixed order. */
srq_status_t srq_rmsnorm_bwd(const void *dy, int64_t ld_dy, const void *r, int64_t ld_r, const void *d_residual, int64_t ld_dres,
                             srq_dtype_t dt, const void *w, srq_dtype_t w_dt, const float *rstd, int64_t rows, int64_t cols,
                             void *dx, int64_t ld_dx, float *dw, void *ws, size_t ws_bytes, void *cuda_stream);

typedef enum { SRQ_SILU = 0, SRQ_GELU = 1 /* tanh form */ } srq_act_t;

/* Gated feed-forward block: both projections, the activation and the product in one kernel.
 *   g = X Wg^T,  u = X Wu^T,  h = act(g) * u          X[T, K], Wg and Wu [F, K] block-coded
 * h (block codes, tile_rows = 1: what the down projection reads) and h_out (h itself, type h_dt) may each be
 * NULL, but not both.  gate and up, if not NULL, receive g and u as block codes (tile_rows = 1): the
 * checkpoints srq_glu_bwd reads, 2 bytes per element instead of 4 or 8.  Wg and Wu share tile_rows.
 * Codes are rounded to nearest (SRQ_RNE). */
srq_status_t srq_glu_fwd(const srq_blocks_t *x, const srq_blocks_t *wg, const srq_blocks_t *wu, int64_t T, int64_t F, int64_t K,
                         srq_act_t act, const srq_blocks_t *h, void *h_out, srq_dtype_t h_dt, int64_t ld_h,
                         const srq_blocks_t *gate, const srq_blocks_t *up, uint32_t *device_status, void *cuda_stream);

/* Its backward pass up to the products, from the checkpoints (g, u as their codes stand for):
 *   dg = dh * u * act'(g),   du = dh * act(g),   h = act(g) * u
 * dh[T, F] has type dt.  Any output may be NULL, all have tile_rows = 1:
 *   dg, du [T, F]        for dX = dg Wg + du Wu (write both into one [T, 2F] matrix, next to each other, where F is
 *                        a multiple of 128, and the sum of the two products is one product)
 *   dg_t, du_t [F, T]    for dWg = dg^T X, dWu = du^T X
 *   h_t [F, T]           for the down projection's dW = dY^T h
 * q->tensor_id, + 1 and + 2 are the threshold streams of dg, du and h under SRQ_SR. */
srq_status_t srq_glu_bwd(const void *dh, srq_dtype_t dt, int64_t ld_dh, const srq_blocks_t *gate, const srq_blocks_t *up,
                         int64_t T, int64_t F, srq_act_t act, const srq_qspec_t *q,
                         const srq_blocks_t *dg, const srq_blocks_t *du, const srq_blocks_t *dg_t, const srq_blocks_t *du_t,
                         const srq_blocks_t *h_t, uint32_t *device_status, void *cuda_stream);

/* Waits for the stream, then returns the device status word of the workspace: SRQ_OK, or the
 * first device-side condition recorded by the calls that used this workspace since its header
 * was last cleared (every entry point clears it when it starts). */
srq_status_t srq_poll_status(void *ws, void *cuda_stream);

/* Host-side planning rule of the product kernel, exposed so that it can be checked without a device:
 * with `tiles` output tiles, `k_blocks` 128-byte blocks along the contraction and `groups` tiles
 * running at a time, tiles [0, *full_tiles) are computed whole and each remaining tile in *splits
 * parts (*splits == 1: nothing is split).  Invalid arguments give 0, 0. */
void srq_plan_splits(int64_t tiles, int32_t k_blocks, int32_t groups, int32_t *full_tiles, int32_t *splits);

/* Self-test of the failure path of the product kernel: enqueues a one-thread kernel that waits, for
 * at most limit_us microseconds (1 .. 1000000), on a barrier that nothing signals.  The wait gives
 * up in the same way the bounded waits of the product kernel do: the status word of ws receives
 * SRQ_ERR_TIMEOUT (read it with srq_poll_status), the kernel returns and the context stays usable. */
srq_status_t srq_selftest_bounded_wait(void *ws, size_t ws_bytes, uint32_t limit_us, void *cuda_stream);

/* Measurement aid, not part of the layer: device-side timing of the product kernel inside whatever
 * sequence of calls the caller runs (a whole layer step), which stream events around a call cannot
 * give because a call enqueues several kernels.  slots is a caller-owned DEVICE array of 2 * n
 * 64-bit words that the caller has initialised to (all ones, zero) pairs: the i-th product launch
 * after this call lowers slots[2 i] to the nanosecond time (%globaltimer) at which its first CTA
 * starts work, after the kernel before it has finished, and raises slots[2 i + 1] to the time its
 * last CTA ends; launches beyond n are not timed.  Two atomics per CTA, nothing else changes.
 * srq_set_product_timer(NULL, 0) switches it off.  The setting is process-wide (all streams and
 * devices): time one stream at a time. */
srq_status_t srq_set_product_timer(uint64_t *slots, int64_t n);

/* Measurement aid, not part of the layer: the issue rate of the tensor pipe for the instruction the
 * products use (tcgen05.mma.cta_group::2.kind::i8, M256 N256 K32).  Every CTA pair of the device
 * multiplies operand blocks that already sit in its shared memory, k_blocks (1 .. 2^22) blocks of 128
 * bytes of contraction, into TMEM; nothing moves through global memory.  *ops (host, optional)
 * receives the integer operations of the launch (2 * 256 * 256 * 128 per pair and block); time the
 * launch on the stream and divide.  This is the ceiling the main loop of the products is compared
 * with: the kind::i8 pipe at the clock the power limit allows, with no data movement at all.  The
 * status word of ws reports a wait that ran out (SRQ_ERR_TIMEOUT), as in the product kernel. */
srq_status_t srq_selftest_mma_rate(void *ws, size_t ws_bytes, int32_t k_blocks, int64_t *ops, void *cuda_stream);

/* Static, human-readable name of a status. */
const char *srq_status_string(srq_status_t s);

/* Number of kernels the library has launched in this process (for launch accounting). */
uint64_t srq_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SRQ_H */
