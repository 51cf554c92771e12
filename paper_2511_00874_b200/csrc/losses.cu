// Losses on the logits: log-probabilities of the targets, the clipped policy loss and the preference loss, and their gradients.
//
// One kernel walks the rows.  A row belongs to one CTA, or to a cluster of up to eight where rows are few.  First walk: running
// maximum m and sum s of e^(z - m) in every thread, joined over the CTA and, through distributed shared memory, over the
// cluster.  Then every thread knows logp, and with it the row's gradient at logp (policy), so that the second walk writes the
// logits' gradient at once; the row is re-read from L2, where the first walk has just brought it, so that HBM sees every logit
// once and its gradient once.  The preference loss needs the log-probabilities of whole answers before its first gradient,
// so there the two walks are two launches with a small kernel over the pairs between them.
//
// Exponentials: e^((x - m) / T) = 2^((x - m) log2(e) / T), the difference first (exact for neighbours, so that large logits cost no
// precision), by the hardware's approximation (2 units); sums in binary32 per thread, at most 16384 terms of 32 partial sums.
#include "train.cuh"

namespace srq {

enum RowMode { ROW_LOGP = 0, ROW_GRAD = 1, ROW_POLICY = 2 };
constexpr float LOG2E = 1.4426950408889634f;
#define SRQ_INF __int_as_float(0x7F800000)

struct RowParams {
    const void* x; int64_t rows, classes, ld;
    const void* targets; int32_t wide;
    float k, inv_t, t;                          // log2(e) / T, 1 / T, T
    int32_t parts;                              // CTAs per row
    uint32_t* status;
    float* logp; float* lse;
    float2* stat;                               // (max, 1 / sum) of each row, instead of lse (ROW_LOGP writes, ROW_GRAD reads)
    const float* dlogp;                         // ROW_GRAD
    void* dx; int64_t ldx;                      // gradient at the logits
    const float* old; const float* advantage; const float* weight; const float* ref;
    float clip_lo, clip_hi, kl;                 // bounds of the ratio
    float* row_loss;
    const void* offsets; int32_t off_wide; int64_t last;      // rows outside offsets[0] .. offsets[last] are left alone; may be null
};

// A row's elements as vectors of 16 bytes at 16-byte boundaries; the first and the last vector may lie partly outside.
template <typename T>
struct RowSpan {
    static constexpr int N = 16 / (int)sizeof(T);
    const T* first;                             // aligned address of vector 0
    int skip;                                   // elements of vector 0 before the row
    int64_t vectors;
    __device__ __forceinline__ RowSpan(const T* row, int64_t n) {
        skip = (int)(((uintptr_t)row & 15u) / sizeof(T));
        first = row - skip;
        vectors = (n + skip + N - 1) / N;
    }
};

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float v[16 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    } else {
        v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
        v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
    }
}
// Vector j of a row of n elements; what lies outside the row reads as minus infinity.
template <typename T>
__device__ __forceinline__ void load_vec(const RowSpan<T>& r, int64_t j, int64_t n, float* v) {
    constexpr int N = RowSpan<T>::N;
    const int64_t c = j * N - r.skip;           // class of the vector's first element
    if (c >= 0 && c + N <= n) {
        unpack<T>(*reinterpret_cast<const uint4*>(r.first + j * N), v);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = c + e >= 0 && c + e < n ? (float)r.first[j * N + e] : -SRQ_INF;
    }
}

// (m, s) of two sets joined: s counts in units of e^m.
__device__ __forceinline__ float2 join(float2 a, float2 b, float k) {
    const float m = fmaxf(a.x, b.x), r = m == -SRQ_INF ? 0.0f : m;
    return make_float2(m, a.y * exp2_fast((a.x - r) * k) + b.y * exp2_fast((b.x - r) * k));
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}

template <typename T, int MODE>
__global__ void __launch_bounds__(512) row_kernel(const RowParams P) {
    pdl_enter();
    constexpr int N = RowSpan<T>::N, U = 32 / N;               // vectors in flight per thread and turn
    __shared__ float2 part[17];
    const int64_t row = blockIdx.x / P.parts;
    const int rank = (int)(blockIdx.x - row * P.parts), tid = threadIdx.x, nt = blockDim.x;
    if (P.offsets) {
        if (row < whole_at(P.offsets, P.off_wide, 0) || row >= whole_at(P.offsets, P.off_wide, P.last)) return;     // the whole cluster
    }
    const int64_t target = whole_at(P.targets, P.wide, row);
    bool counts = target >= 0 && target < P.classes;
    if (target >= P.classes && tid == 0 && rank == 0) note(P.status, SRQ_ERR_INVALID_ARG);
    float weight = 1.0f, old = 0.0f, adv = 0.0f, ref = 0.0f, c = 0.0f;
    if constexpr (MODE == ROW_POLICY) {
        weight = P.weight[row];
        counts = counts && weight != 0.0f;
        if (counts) { old = P.old[row]; adv = P.advantage[row]; if (P.ref) ref = P.ref[row]; }
    }
    const T* x = reinterpret_cast<const T*>(P.x) + row * P.ld;
    const RowSpan<T> span(x, P.classes);
    const int64_t share = (span.vectors + P.parts - 1) / P.parts, j0 = rank * share, j1 = j0 + share < span.vectors ? j0 + share : span.vectors;
    float m = -SRQ_INF, inv = 0.0f;
    if constexpr (MODE == ROW_GRAD) {
        c = counts ? P.dlogp[row] : 0.0f;
        if (c != 0.0f) {
            if (P.stat) { const float2 q = P.stat[row]; m = q.x; inv = q.y; }
            else { m = P.lse[row] * P.t; inv = 1.0f; }
        }
    } else {
        const float xt = counts ? (float)x[target] : 0.0f;
        float2 all = make_float2(0.0f, 1.0f);
        if (counts) {
            float s0 = 0.0f, s1 = 0.0f;
            for (int64_t j = j0 + tid; j < j1; j += (int64_t)nt * U) {
                float v[U * N];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (j + (int64_t)u * nt < j1) load_vec<T>(span, j + (int64_t)u * nt, P.classes, v + u * N);
                    else
#pragma unroll
                        for (int e = 0; e < N; ++e) v[u * N + e] = -SRQ_INF;
                }
                float top = m;
#pragma unroll
                for (int e = 0; e < U * N; ++e) top = fmaxf(top, v[e]);
                const float r = top == -SRQ_INF ? 0.0f : top, f = exp2_fast((m - r) * P.k);
                s0 *= f; s1 *= f; m = top;
#pragma unroll
                for (int e = 0; e < U * N; e += 2) {
                    const float2 d = __fmul2_rn(__fadd2_rn(make_float2(v[e], v[e + 1]), make_float2(-r, -r)), make_float2(P.k, P.k));
                    s0 += exp2_fast(d.x); s1 += exp2_fast(d.y);
                }
            }
            all = make_float2(m, s0 + s1);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const float2 o = make_float2(__shfl_xor_sync(0xFFFFFFFFu, all.x, d), __shfl_xor_sync(0xFFFFFFFFu, all.y, d));
            all = join(all, o, P.k);
        }
        if ((tid & 31) == 0) part[tid >> 5] = all;
        __syncthreads();
        all = part[0];
        for (int w = 1; w < nt / 32; ++w) all = join(all, part[w], P.k);
        if (P.parts > 1) {
            if (tid == 0) part[16] = all;
            cluster_sync();
            float2 sum = make_float2(-SRQ_INF, 0.0f);
            for (int q = 0; q < P.parts; ++q) {
                float2 o;
                asm volatile("{\n.reg .u32 a;\nmapa.shared::cluster.u32 a, %2, %3;\nld.shared::cluster.v2.f32 {%0, %1}, [a];\n}"
                             : "=f"(o.x), "=f"(o.y) : "r"((uint32_t)__cvta_generic_to_shared(&part[16])), "r"(q) : "memory");
                sum = join(sum, o, P.k);
            }
            all = sum;
            cluster_sync();                                    // nobody leaves while its sums are being read
        }
        m = all.x; inv = 1.0f / all.y;
        const float log_s = logf(all.y), logp = counts ? (xt - m) * P.inv_t - log_s : 0.0f;
        float loss = 0.0f;
        if constexpr (MODE == ROW_POLICY) {
            if (counts) {
                const float rho = expf(logp - old), a = rho * adv, b = fminf(fmaxf(rho, P.clip_lo), P.clip_hi) * adv;
                loss = a <= b ? -a : -b;
                c = a <= b ? -a : 0.0f;
                if (a != a) loss = c = a;                      // NaN stays NaN
                if (P.ref) {
                    const float d = ref - logp, g = expm1f(d);
                    loss += P.kl * (g - d);
                    c -= P.kl * g;
                }
                loss *= weight; c *= weight;
            }
        }
        if (tid == 0 && rank == 0) {
            if (P.logp) P.logp[row] = logp;
            if (P.lse) P.lse[row] = counts ? m * P.inv_t + log_s : 0.0f;
            if (P.stat) P.stat[row] = make_float2(m, inv);
            if constexpr (MODE == ROW_POLICY) if (P.row_loss) P.row_loss[row] = loss;
            if (abs_word(logp) >= 0x7F800000u || abs_word(c) >= 0x7F800000u) note(P.status, SRQ_ERR_NONFINITE);
        }
    }
    if constexpr (MODE != ROW_LOGP) {
        if (!P.dx) return;
        T* y = reinterpret_cast<T*>(P.dx) + row * P.ldx;
        c *= P.inv_t;
        const float f = -c * inv;
        const bool same = (((uintptr_t)y ^ (uintptr_t)x) & 15u) == 0;
        T* y0 = y - span.skip;                                 // where vector 0 would begin
        for (int64_t j = j0 + tid; j < j1; j += (int64_t)nt * U) {
            float v[U * N];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = j + (int64_t)u * nt;
                if (c != 0.0f && i < j1) load_vec<T>(span, i, P.classes, v + u * N);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = j + (int64_t)u * nt;
                if (i >= j1) break;
                float* w = v + u * N;
                const int64_t first = i * N - span.skip;
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    if (c != 0.0f) {
                        const float2 d = __fmul2_rn(__fadd2_rn(make_float2(w[e], w[e + 1]), make_float2(-m, -m)), make_float2(P.k, P.k));
                        const float2 p = __fmul2_rn(make_float2(exp2_fast(d.x), exp2_fast(d.y)), make_float2(f, f));
                        w[e] = p.x; w[e + 1] = p.y;
                    } else { w[e] = 0.0f; w[e + 1] = 0.0f; }
                }
                if (target >= first && target < first + N) {
#pragma unroll
                    for (int e = 0; e < N; ++e) if (first + e == target) w[e] += c;
                }
                if (same && first >= 0 && first + N <= P.classes) {
                    uint4 o;
                    if constexpr (sizeof(T) == 4) {
                        o = make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
                    } else {
                        uint32_t q[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(w[2 * e], w[2 * e + 1]);
                            q[e] = *reinterpret_cast<const uint32_t*>(&b);
                        }
                        o = make_uint4(q[0], q[1], q[2], q[3]);
                    }
                    *reinterpret_cast<uint4*>(y0 + i * N) = o;
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) if (first + e >= 0 && first + e < P.classes) y0[i * N + e] = (T)w[e];
                }
            }
        }
    }
}

// out[0] = scale * sum of x[0 .. n): one CTA, binary64, a fixed order.
__global__ void __launch_bounds__(1024) loss_sum_kernel(const float* x, int64_t n, double scale, float* out) {
    pdl_enter();
    __shared__ double part[32];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += (double)x[i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = part[threadIdx.x];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        if (threadIdx.x == 0) out[0] = (float)(s * scale);
    }
}

struct PairParams {
    const float* logp; const float* ref; const void* targets; int32_t wide;
    const void* offsets; int32_t off_wide; int64_t rows, classes, pairs;
    float beta, smoothing;
    float* pair_loss; float* dlogp;
    uint32_t* status;
};

// One CTA per pair: both answers' sums, the pair's loss and the gradient at every logp of the two.
__global__ void __launch_bounds__(256) pair_kernel(const PairParams P) {
    pdl_enter();
    __shared__ double part[8];
    const int tid = threadIdx.x;
    const int64_t i = blockIdx.x;
    const int64_t a = whole_at(P.offsets, P.off_wide, 2 * i), b = whole_at(P.offsets, P.off_wide, 2 * i + 1), e = whole_at(P.offsets, P.off_wide, 2 * i + 2);
    if (!(0 <= a && a <= b && b <= e && e <= P.rows)) {
        if (tid == 0) { note(P.status, SRQ_ERR_INVALID_ARG); P.pair_loss[i] = 0.0f; }
        return;
    }
    double s = 0.0;
    for (int64_t r = a + tid; r < e; r += 256) {
        const int64_t t = whole_at(P.targets, P.wide, r);
        if (t < 0 || t >= P.classes) continue;
        const double d = (double)P.logp[r] - (double)P.ref[r];
        s += r < b ? d : -d;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if ((tid & 31) == 0) part[tid >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w];
    const float h = (float)(s * (double)P.beta);
    // -log sigma(h) = max(-h, 0) + log(1 + e^-|h|);  sigma(-h) = 1 / (1 + e^h)
    const float tail = log1pf(expf(-fabsf(h)));
    const float loss = (1.0f - P.smoothing) * (fmaxf(-h, 0.0f) + tail) + P.smoothing * (fmaxf(h, 0.0f) + tail);
    const float dh = P.smoothing - 1.0f / (1.0f + expf(h));
    if (tid == 0) {
        P.pair_loss[i] = h != h ? h : loss;
        if (abs_word(h) >= 0x7F800000u) note(P.status, SRQ_ERR_NONFINITE);
    }
    const float c = dh * P.beta / (float)P.pairs;
    for (int64_t r = a + tid; r < e; r += 256) P.dlogp[r] = r < b ? c : -c;
}

// CTAs per row and threads per CTA: one CTA a row where rows fill the device, up to a cluster of eight where they do not and
// the row is long enough to share.
static void row_shape(int64_t rows, int64_t vectors, int* parts, int* threads) {
    const int sms = sm_count();
    int p = 1;
    while (p < 8 && rows * p < 2 * (int64_t)sms && vectors >= 512 * (int64_t)p) p <<= 1;
    const int64_t share = vectors / p;
    *parts = p;
    *threads = share >= 1024 ? 512 : share >= 512 ? 256 : 128;
}

template <typename T, int MODE>
static cudaError_t launch_rows(RowParams P, cudaStream_t st) {
    int threads;
    row_shape(P.rows, (P.classes * (int64_t)sizeof(T) + 15) / 16, &P.parts, &threads);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(P.rows * P.parts)); cfg.blockDim = dim3(threads); cfg.stream = st;
    cudaLaunchAttribute at[2];
    int n = 0;
    if (P.parts > 1 && MODE != ROW_GRAD) {                     // the gradient's walk exchanges nothing
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = (unsigned)P.parts; at[n].val.clusterDim.y = 1; at[n].val.clusterDim.z = 1;
        ++n;
    }
    if (pdl_allowed(st)) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = at; cfg.numAttrs = n;
    count_launch();
    return cudaLaunchKernelEx(&cfg, row_kernel<T, MODE>, P);
}
template <int MODE>
static cudaError_t launch_rows(const RowParams& P, int32_t dt, cudaStream_t st) {
    return dt == SRQ_F32 ? launch_rows<float, MODE>(P, st) : launch_rows<__nv_bfloat16, MODE>(P, st);
}

static RowParams row_params(const LogitsArgs& a) {
    RowParams P = {};
    P.x = a.x; P.rows = a.rows; P.classes = a.classes; P.ld = a.ld;
    P.targets = a.targets; P.wide = a.target_t == SRQ_I64;
    P.k = LOG2E / a.temperature; P.inv_t = 1.0f / a.temperature; P.t = a.temperature;
    P.status = a.status;
    return P;
}

cudaError_t launch_logprob_fwd(const LogitsArgs& a, float* logp, float* lse, cudaStream_t st) {
    RowParams P = row_params(a);
    P.logp = logp; P.lse = lse;
    return launch_rows<ROW_LOGP>(P, a.dt, st);
}
cudaError_t launch_logprob_bwd(const LogitsArgs& a, const float* lse, const float* dlogp, void* dx, int64_t ldx, cudaStream_t st) {
    RowParams P = row_params(a);
    P.lse = const_cast<float*>(lse); P.dlogp = dlogp; P.dx = dx; P.ldx = ldx;
    return launch_rows<ROW_GRAD>(P, a.dt, st);
}
static cudaError_t launch_loss_sum(const float* x, int64_t n, double scale, float* out, cudaStream_t st) {
    count_launch();
    return launch_pdl(loss_sum_kernel, dim3(1), dim3(1024), 0, st, x, n, scale, out);
}
cudaError_t launch_policy(const LogitsArgs& a, const PolicyArgs& p, cudaStream_t st) {
    RowParams P = row_params(a);
    P.logp = p.logp; P.dx = p.dx; P.ldx = p.ldx; P.old = p.old; P.advantage = p.advantage; P.weight = p.weight; P.ref = p.ref;
    P.clip_lo = 1.0f - p.h.clip_low; P.clip_hi = 1.0f + p.h.clip_high; P.kl = p.h.kl_coef; P.row_loss = p.row_loss;
    const cudaError_t e = launch_rows<ROW_POLICY>(P, a.dt, st);
    if (e != cudaSuccess || !p.loss) return e;
    return launch_loss_sum(p.row_loss, a.rows, 1.0, p.loss, st);
}

// Workspace: (max, 1 / sum) and the gradient at logp of every row.
size_t preference_bytes(int64_t rows) { return align_up((size_t)rows * 8) + align_up((size_t)rows * 4); }

cudaError_t launch_preference(const LogitsArgs& a, const PreferenceArgs& p, void* ws, cudaStream_t st) {
    RowParams P = row_params(a);
    P.stat = reinterpret_cast<float2*>(ws);
    float* dlogp = reinterpret_cast<float*>((char*)ws + align_up((size_t)a.rows * 8));
    P.logp = p.logp; P.offsets = p.offsets; P.off_wide = p.offset_t == SRQ_I64; P.last = 2 * p.pairs;
    cudaError_t e = a.rows ? launch_rows<ROW_LOGP>(P, a.dt, st) : cudaSuccess;
    if (e != cudaSuccess) return e;
    PairParams Q = {};
    Q.logp = p.logp; Q.ref = p.ref; Q.targets = a.targets; Q.wide = P.wide; Q.offsets = p.offsets; Q.off_wide = P.off_wide;
    Q.rows = a.rows; Q.classes = a.classes; Q.pairs = p.pairs; Q.beta = p.h.beta; Q.smoothing = p.h.label_smoothing;
    Q.pair_loss = p.pair_loss; Q.dlogp = dlogp; Q.status = a.status;
    e = launch_pdl(pair_kernel, dim3((unsigned)p.pairs), dim3(256), 0, st, Q);
    count_launch();
    if (e != cudaSuccess) return e;
    if (p.dx && a.rows) {
        P.dlogp = dlogp; P.dx = p.dx; P.ldx = p.ldx; P.logp = nullptr;
        e = launch_rows<ROW_GRAD>(P, a.dt, st);
        if (e != cudaSuccess) return e;
    }
    return p.loss ? launch_loss_sum(p.pair_loss, p.pairs, 1.0 / (double)p.pairs, p.loss, st) : cudaSuccess;
}

}  // namespace srq
