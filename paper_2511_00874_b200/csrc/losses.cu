// Losses on the logits: log-probabilities of the targets, the clipped policy loss and the preference loss, and their gradients.
//
// One kernel walks the rows.  A row belongs to one CTA, or to a cluster of up to eight that shares it.  Every thread copies its
// vectors of the row into shared memory, several groups ahead of the one it works on (cp.async; a thread reads only what it has copied
// itself, so that nothing but its own copies is waited for).  First walk: running maximum and sum of the exponentials, joined
// over the CTA and, through distributed shared memory, over the cluster.  Then every thread knows logp, and with it the row's gradient at logp
// (policy), so that the second walk writes the logits' gradient at once, from shared memory where the row's share fits there (up to 32 KB
// per CTA, 256 KB per row), else by copying it once more, mostly out of L2: HBM sees every logit once and its gradient once.  The
// preference loss needs the log-probabilities of whole answers before its first gradient, so there the two walks are two
// launches with a small kernel over the pairs between them.
//
// Bound: HBM at best (2 bytes in, 2 bytes out per bfloat16 logit); what keeps the policy loss from it is that a row's phases follow one another
// (flags, copies, sums, the cluster's barrier, gradient) and six CTAs per SM do not cover all of them, with two exponentials per logit taking
// 0.6 of their pipe's cycles.  Policy loss, 4096 x 131072 bfloat16, an eighth of the rows masked: 381 - 423 us = 4.8 - 5.3 TB/s; 1021 x 50257
// binary32: 78 - 81 us = 4.9 - 5.0 TB/s.  Preference loss, 8044 rows x 50257 bfloat16: 388 - 430 us on different machines; where it took 388,
// 140 were for the sums (5.8 TB/s) and 242 for the gradient (6.7 TB/s, some of it out of L2).  A persistent form that copied the next row
// meanwhile was slower (608 us: two large CTAs fewer per SM to cover the barriers, and clusters of eight that do not fill the device).
//
// Exponentials: e^((x - m) / T) = 2^((x - m) k) with k = log2(e) / T, the difference first, so that large logits cost no precision
// and the range is binary32's (a gradient that is given lse alone: LSE_EXACT below).  k is a sum of two numbers where probabilities
// are added up (one alone would shift every log-probability of a row the same way, which shows in sums over rows).  2^y is the
// hardware's approximation (2 units).  Sums are binary32: a thread has two, of at most classes / 256 terms each where a row is one
// CTA's (512 at 131072 classes), and their joins follow.
#include <float.h>
#include <math.h>

#include "train.cuh"

namespace srq {

// ROW_GRAD: the gradient from (max, 1 / sum) of every row; ROW_LSE: from lse, where that is exact enough, else the row is walked twice as for
// ROW_POLICY.
enum RowMode { ROW_LOGP = 0, ROW_GRAD = 1, ROW_POLICY = 2, ROW_LSE = 3 };
// A gradient from one binary32 number for maximum and sum takes lse's rounding as an error of every exponent, 2^-24 |lse|: up to this |lse| it
// is what a difference x - max of that size costs anyway (relative error of a probability: a few 1e-6).  Beyond, at 1e4 it would be 6e-4, at 1e8
// probabilities of a row no longer add up to anything near 1.  The logits of a model at temperature 1 have an lse of 5 to 30.
// (8044 x 50257 bfloat16: 258 us from lse, 334 walked twice; 1021 x 50257 binary32: 71 and 86.)
constexpr float LSE_EXACT = 32.0f;
#define SRQ_INF __int_as_float(0x7F800000)

struct RowParams {
    const void* x; int64_t rows, classes, ld;
    const void* targets; int32_t wide;
    float k, k_low, inv_t, t;                   // log2(e) / T and what it lacks, 1 / T, T
    int32_t parts;                              // CTAs per row
    uint32_t* status;
    float* logp; float* lse;
    float2* stat;                               // (max, 1 / sum) of each row (ROW_LOGP writes, ROW_GRAD reads)
    const float* dlogp;                         // ROW_GRAD, ROW_LSE
    void* dx; int64_t ldx;                      // gradient at the logits
    const float* old; const float* advantage; const float* weight; const float* ref;
    float clip_lo, clip_hi, kl;                 // bounds of the ratio
    float* row_loss;
    const void* offsets; int32_t off_wide; int64_t last;      // rows outside offsets[0] .. offsets[last] are left alone; may be null
    int32_t clear_rest;                         // or do not count
};

// A row's elements as vectors of 16 bytes at 16-byte boundaries; the first and the last vector may lie partly outside.
template <typename T>
struct RowSpan {
    static constexpr int N = 16 / (int)sizeof(T);
    const T* first;                             // aligned address of vector 0
    int skip, n;                                // elements of vector 0 before the row, classes
    int vectors, lo, hi;                        // vectors; those that lie wholly inside: lo .. hi - 1
    __device__ __forceinline__ RowSpan(const T* row, int64_t classes) {
        n = (int)classes;
        skip = (int)(((uintptr_t)row & 15u) / sizeof(T));
        first = row - skip;
        vectors = (int)((classes + skip + N - 1) / N);
        lo = skip ? 1 : 0;
        hi = (int)((classes + skip) / N);
    }
    __device__ __forceinline__ bool inside(int j) const { return j >= lo && j < hi; }
    __device__ __forceinline__ int64_t element(int j) const { return (int64_t)j * N - skip; }      // class of vector j's first element
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
// Copies vector j of a row to dst; what lies outside the row becomes minus infinity.
template <typename T>
__device__ __forceinline__ void copy_vec(const RowSpan<T>& r, int j, uint4* dst) {
    constexpr int N = RowSpan<T>::N;
    const T* src = r.first + (int64_t)j * N;
    if (r.inside(j)) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
    } else {
        const int64_t c = r.element(j);
        T* d = reinterpret_cast<T*>(dst);
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = c + e >= 0 && c + e < r.n ? src[e] : (T)-SRQ_INF;
    }
}

// 2^(d k) of two differences.
__device__ __forceinline__ float2 powers(float2 d, float2 k, float2 k_low) {
    const float2 t = __ffma2_rn(d, k_low, __fmul2_rn(d, k));
    return make_float2(exp2_fast(t.x), exp2_fast(t.y));
}
// The cluster's barrier without an order of memory: whoever has written for others fences first.  Both halves take converged warps.
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A thread's vectors first, first + NT, ... of a row (NT: threads of the CTA), by way of shared memory: the thread's i-th in its slot i % ROW_SLOTS.
// ROW_GROUP vectors are copied and waited for together, ROW_AHEAD groups ahead.
constexpr int ROW_GROUP = 2, ROW_AHEAD = 8, ROW_SLOTS = ROW_GROUP * ROW_AHEAD;
// Waits until at most n groups of copies are on their way (n: a constant once loops are unrolled).
__device__ __forceinline__ void wait_copies(int n) {
    switch (n) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
        case 5: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
        case 6: asm volatile("cp.async.wait_group 6;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 7;" ::: "memory"); break;
    }
}
static_assert(ROW_AHEAD <= 8, "wait_copies");

// Groups that are complete and wholly inside the row for all lanes of a warp are plain: one comparison that is the same for the warp
// decides, and nothing of a plain group is checked (with a check per vector and lane a third of all instructions were checks).
template <typename T, int NT>
struct RowStream {
    static constexpr int GROUP_BYTES = ROW_GROUP * NT * 16;
    const RowSpan<T>& span;
    int first, count;                           // the thread's first vector, how many
    int groups, plain_lo, plain_hi;             // of the warp: groups, the plain ones are plain_lo .. plain_hi - 1
    uint4* buffer;                              // the thread's first slot
    __device__ __forceinline__ RowStream(const RowSpan<T>& s, int j0, int j1, uint4* staged) : span(s) {
        first = j0 + (int)threadIdx.x;
        count = first < j1 ? (j1 - first + NT - 1) / NT : 0;
        buffer = staged + threadIdx.x;
        const int in = first < s.hi ? (s.hi - first + NT - 1) / NT : 0;        // vectors before the end of those inside
        groups = __reduce_max_sync(0xFFFFFFFFu, (count + ROW_GROUP - 1) / ROW_GROUP);
        plain_lo = __reduce_max_sync(0xFFFFFFFFu, first >= s.lo ? 0 : 1);
        plain_hi = __reduce_min_sync(0xFFFFFFFFu, (in < count ? in : count) / ROW_GROUP);
    }
    __device__ __forceinline__ int vector(int i) const { return first + i * NT; }
    __device__ __forceinline__ bool plain(int g) const { return g >= plain_lo && g < plain_hi; }
    // group g of the row to the slots at `slot`, as far as there is such a group; closes the copies' group
    __device__ __forceinline__ void copy_group(int g, uint4* slot) const {
        if (plain(g)) {
            const char* src = reinterpret_cast<const char*>(span.first) + (int64_t)first * 16 + (int64_t)g * GROUP_BYTES;
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(slot);
#pragma unroll
            for (int u = 0; u < ROW_GROUP; ++u)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + u * NT * 16), "l"(src + u * NT * 16) : "memory");
        } else if (g < groups) {
#pragma unroll 1
            for (int u = 0; u < ROW_GROUP && g * ROW_GROUP + u < count; ++u) copy_vec<T>(span, vector(g * ROW_GROUP + u), slot + u * NT);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ bool resident() const { return groups <= ROW_AHEAD; }
    // fast(g, slot) for plain groups, slow(g, slot) for the others: the vectors of group g are in slot[0], slot[NT], ...  copy: they have to be
    // brought there.  Where all groups have slots of their own the plain ones come first, in straight code.
    template <typename Fast, typename Slow>
    __device__ __forceinline__ void walk(bool copy, Fast&& fast, Slow&& slow) const {
        if (copy) {
#pragma unroll
            for (int g = 0; g < ROW_AHEAD; ++g) copy_group(g, buffer + g * ROW_GROUP * NT);
        }
        if (resident()) {
#pragma unroll
            for (int g = 0; g < ROW_AHEAD; ++g) {
                if (copy) wait_copies(ROW_AHEAD - 1 - g);
                if (plain(g)) fast(g, buffer + g * ROW_GROUP * NT);
            }
#pragma unroll 1
            for (int g = 0; g < groups; ++g)
                if (!plain(g)) slow(g, buffer + g * ROW_GROUP * NT);
            return;
        }
#pragma unroll 1
        for (int g = 0, at = 0; g < groups; ++g) {
            uint4* slot = buffer + at;
            at = at == (ROW_AHEAD - 1) * ROW_GROUP * NT ? 0 : at + ROW_GROUP * NT;
            if (copy) wait_copies(ROW_AHEAD - 1);
            if (plain(g)) fast(g, slot); else slow(g, slot);
            if (copy) copy_group(g + ROW_AHEAD, slot);
        }
    }
};

// One vector's gradient: f 2^((x - m) k).
template <typename T>
__device__ __forceinline__ void gradient(const uint4& raw, float m, float2 k2, float2 low2, float f, float w[16 / sizeof(T)]) {
    unpack<T>(raw, w);
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); e += 2) {
        const float2 d = __fadd2_rn(make_float2(w[e], w[e + 1]), make_float2(-m, -m));
        const float2 z = sizeof(T) == 4 ? __ffma2_rn(d, low2, __fmul2_rn(d, k2)) : __fmul2_rn(d, k2);   // (k_low: lost in a bfloat16 result's rounding)
        const float2 p = __fmul2_rn(make_float2(exp2_fast(z.x), exp2_fast(z.y)), make_float2(f, f));
        w[e] = p.x; w[e + 1] = p.y;
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float w[16 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
    else {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(w[2 * e], w[2 * e + 1]);
            q[e] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(q[0], q[1], q[2], q[3]);
    }
}

// CTAs of NT threads per SM that registers are kept for: what shared memory allows with 32 KB each, and sixteen of a warp.
template <int NT> constexpr int ROW_CTAS = NT == 128 ? 6 : 16;

// What the second walk needs of a row: the maximum, 1 / sum, the gradient at logp.
struct RowResult { float m, inv, c; };

template <typename T, int MODE, int NT>
__global__ void __launch_bounds__(NT, ROW_CTAS<NT>) row_kernel(const RowParams P) {
    pdl_enter();
    constexpr int N = RowSpan<T>::N;
    extern __shared__ uint4 staged[];
    __shared__ float2 part[NT / 32], mine;
    __shared__ RowResult shared_result;
    int64_t row = blockIdx.x / P.parts;
    const int rank = (int)(blockIdx.x - row * P.parts), tid = threadIdx.x;
    // the second walk over the same logits begins with the rows that the first one read last: some are still in L2
    if (MODE == ROW_GRAD) row = P.rows - 1 - row;
    bool rest = false;
    if (P.offsets) {
        rest = row < whole_at(P.offsets, P.off_wide, 0) || row >= whole_at(P.offsets, P.off_wide, P.last);
        if (rest && !P.clear_rest) return;                     // the whole cluster
    }
    const int64_t target = rest ? -1 : whole_at(P.targets, P.wide, row);
    bool counts = target >= 0 && target < P.classes;
    if (target >= P.classes && tid == 0 && rank == 0) note(P.status, SRQ_ERR_INVALID_ARG);
    float weight = 1.0f;
    if constexpr (MODE == ROW_POLICY) {
        weight = P.weight[row];
        counts = counts && weight != 0.0f;
    }
    const T* x = reinterpret_cast<const T*>(P.x) + row * P.ld;
    const RowSpan<T> span(x, P.classes);
    const int share = (span.vectors + P.parts - 1) / P.parts, j0 = rank * share, j1 = j0 + share < span.vectors ? j0 + share : span.vectors;
    const RowStream<T, NT> stream(span, j0, j1, staged);
    const float2 k2 = make_float2(P.k, P.k), low2 = make_float2(P.k_low, P.k_low);
    RowResult r = {0.0f, 0.0f, 0.0f};
    bool sums = MODE == ROW_LOGP || MODE == ROW_POLICY;        // the first walk takes place (the same for the whole cluster)
    if constexpr (MODE == ROW_GRAD || MODE == ROW_LSE) {
        r.c = counts ? P.dlogp[row] : 0.0f;
        if (r.c != 0.0f) {
            if constexpr (MODE == ROW_GRAD) {
                const float2 q = P.stat[row];
                r.m = q.x; r.inv = q.y;
            } else {
                const float lse = P.lse[row];
                r.m = lse * P.t; r.inv = 1.0f;
                sums = !(fabsf(lse) <= LSE_EXACT);             // (or lse is not finite, though the row's probabilities may be)
            }
        }
    }
    if (MODE != ROW_GRAD && sums) {
        // what the row's first warp will need, requested before the walk
        float xt = 0.0f, old = 0.0f, adv = 0.0f, ref = 0.0f;
        if (MODE != ROW_LSE && counts && tid < 32) {
            xt = (float)x[target];
            if constexpr (MODE == ROW_POLICY) { old = P.old[row]; adv = P.advantage[row]; if (P.ref) ref = P.ref[row]; }
        }
        float m = -SRQ_INF;
        float2 sum = make_float2(0.0f, 0.0f);
        if (counts) {
            const auto add = [&](const float v[ROW_GROUP * N]) {
                float top = m;
#pragma unroll
                for (int e = 0; e < ROW_GROUP * N; ++e) top = fmaxf(top, v[e]);
                const float to = top == -SRQ_INF ? 0.0f : top, f = exp2_fast((m - to) * P.k);
                sum = __fmul2_rn(sum, make_float2(f, f));
                m = top;
#pragma unroll
                for (int e = 0; e < ROW_GROUP * N; e += 2)
                    sum = __fadd2_rn(sum, powers(__fadd2_rn(make_float2(v[e], v[e + 1]), make_float2(-to, -to)), k2, low2));
            };
            stream.walk(true, [&](int, const uint4* slot) {
                uint4 raw[ROW_GROUP];
                float v[ROW_GROUP * N];
#pragma unroll
                for (int u = 0; u < ROW_GROUP; ++u) raw[u] = slot[u * NT];
#pragma unroll
                for (int u = 0; u < ROW_GROUP; ++u) unpack<T>(raw[u], v + u * N);
                add(v);
            }, [&](int g, const uint4* slot) {
                float v[ROW_GROUP * N];
#pragma unroll
                for (int u = 0; u < ROW_GROUP; ++u) {
                    if (g * ROW_GROUP + u < stream.count) unpack<T>(slot[u * NT], v + u * N);
                    else
#pragma unroll
                        for (int e = 0; e < N; ++e) v[u * N + e] = -SRQ_INF;
                }
                add(v);
            });
        }
        // (m, s) of the warp, the CTA and the cluster: the largest m first, then the sums in its units
        float s = sum.x + sum.y;
        const auto reduce = [&](int lanes) {
            float top = m;
            for (int d = lanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            s *= exp2_fast((m - (top == -SRQ_INF ? 0.0f : top)) * P.k);
            m = top;
            for (int d = lanes / 2; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        };
        reduce(32);
        if constexpr (NT > 32) {
            if ((tid & 31) == 0) part[tid >> 5] = make_float2(m, s);
            __syncthreads();
            if (tid < 32) {
                const float2 o = tid < NT / 32 ? part[tid] : make_float2(-SRQ_INF, 0.0f);
                m = o.x; s = o.y;
                reduce(NT / 32);
            }
        }
        if (P.parts > 1) {
            if (tid == 0) {
                mine = make_float2(m, s);
                asm volatile("fence.acq_rel.cluster;" ::: "memory");
            }
            cluster_arrive();
            cluster_wait();
            if (tid < 32) {
                m = -SRQ_INF; s = 0.0f;
                if (tid < P.parts)
                    asm volatile("{\n.reg .u32 a;\nmapa.shared::cluster.u32 a, %2, %3;\nld.shared::cluster.v2.f32 {%0, %1}, [a];\n}"
                                 : "=f"(m), "=f"(s) : "r"((uint32_t)__cvta_generic_to_shared(&mine)), "r"(tid) : "memory");
                reduce(8);
            }
        }
        if (tid < 32) {                                        // (lane 0 holds the sums)
            r.m = m; r.inv = 1.0f / s;
            const float log_s = logf(s), logp = counts ? (xt - m) * P.inv_t - log_s : 0.0f, lse = counts ? m * P.inv_t + log_s : 0.0f;
            float loss = 0.0f;
            if constexpr (MODE == ROW_POLICY) {
                if (counts) {
                    float rho = expf(logp - old);
                    if (adv == 0.0f && rho == SRQ_INF) rho = FLT_MAX;          // the ratio is finite, and so its product with 0 is 0
                    const float a = rho * adv, b = fminf(fmaxf(rho, P.clip_lo), P.clip_hi) * adv;
                    loss = a <= b ? -a : -b;
                    r.c = a <= b ? -a : 0.0f;
                    if (a != a) loss = r.c = a;                // NaN stays NaN
                    if (P.ref) {
                        const float d = ref - logp, g = expm1f(d);
                        loss += P.kl * (g - d);
                        r.c -= P.kl * g;
                    }
                    loss *= weight; r.c *= weight;
                }
            }
            if (tid == 0) {
                shared_result = r;
                if (MODE != ROW_LSE && rank == 0) {
                    if (P.logp) P.logp[row] = logp;
                    if (MODE == ROW_LOGP && P.lse) {
                        P.lse[row] = lse;
                        if (abs_word(lse) >= 0x7F800000u) note(P.status, SRQ_ERR_NONFINITE);
                    }
                    if (P.stat) P.stat[row] = make_float2(m, r.inv);
                    if constexpr (MODE == ROW_POLICY) if (P.row_loss) P.row_loss[row] = loss;
                    if (abs_word(logp) >= 0x7F800000u || abs_word(r.c) >= 0x7F800000u || (P.row_loss && abs_word(loss) >= 0x7F800000u)) note(P.status, SRQ_ERR_NONFINITE);
                }
            }
        }
        __syncthreads();
        if (P.parts > 1) cluster_arrive();                     // no CTA leaves while its sums are being read: the wait is at the end
        r = shared_result;
    }
    if constexpr (MODE != ROW_LOGP) {
        if (P.dx) {
            T* y = reinterpret_cast<T*>(P.dx) + row * P.ldx;
            const float c = r.c * P.inv_t, f = -c * r.inv;
            const bool same = (((uintptr_t)y ^ (uintptr_t)x) & 15u) == 0, zero = c == 0.0f;
            T* y0 = y - span.skip;                             // where vector 0 would begin
            // The target's vector is written like the others, and its thread writes the target's element once more, last.
            const int away = counts ? (int)((target + span.skip) / N) - stream.first : -1, target_i = away >= 0 && away % NT == 0 ? away / NT : -1;
            const bool has_target = target_i >= 0 && target_i < stream.count;
            float at_target = c;
            if (has_target && !zero) at_target = c + f * powers(make_float2((float)x[target] - r.m, 0.0f), k2, low2).x;      // (before it is overwritten)
            const auto some = [&](int g, const uint4* slot) {
#pragma unroll 1
                for (int u = 0; u < ROW_GROUP && g * ROW_GROUP + u < stream.count; ++u) {
                    const int j = stream.vector(g * ROW_GROUP + u);
                    float w[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) w[e] = 0.0f;
                    if (!zero) gradient<T>(slot[u * NT], r.m, k2, low2, f, w);
                    if (same && span.inside(j)) {
                        *reinterpret_cast<uint4*>(y0 + (int64_t)j * N) = pack<T>(w);
                    } else {
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const int64_t col = span.element(j) + e;
                            if (col >= 0 && col < P.classes) y[col] = (T)w[e];
                        }
                    }
                }
            };
            const bool copy = !zero && !(MODE != ROW_GRAD && sums && stream.resident());
            if (!same) {                                       // nothing of the gradient's row is aligned as the logits' is
                stream.walk(copy, some, some);
            } else if (zero) {
                stream.walk(false, [&](int g, const uint4*) {
                    uint4* out = reinterpret_cast<uint4*>(y0 + (int64_t)stream.first * N + (int64_t)g * (ROW_GROUP * NT * N));
#pragma unroll
                    for (int u = 0; u < ROW_GROUP; ++u) out[u * NT] = make_uint4(0, 0, 0, 0);
                }, some);
            } else {
                stream.walk(copy, [&](int g, const uint4* slot) {
                    uint4* out = reinterpret_cast<uint4*>(y0 + (int64_t)stream.first * N + (int64_t)g * (ROW_GROUP * NT * N));
                    uint4 raw[ROW_GROUP];
#pragma unroll
                    for (int u = 0; u < ROW_GROUP; ++u) raw[u] = slot[u * NT];
#pragma unroll
                    for (int u = 0; u < ROW_GROUP; ++u) {
                        float w[N];
                        gradient<T>(raw[u], r.m, k2, low2, f, w);
                        out[u * NT] = pack<T>(w);
                    }
                }, some);
            }
            if (has_target && !zero) y[target] = (T)at_target;
        }
    }
    if (MODE != ROW_GRAD && sums && P.parts > 1) cluster_wait();
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

// -log sigma(h) = max(-h, 0) + log(1 + e^-|h|);  sigma(-h) = 1 / (1 + e^h)
__device__ __forceinline__ float pair_loss_of(float h, float smoothing) {
    if (h != h) return h;
    const float tail = log1pf(expf(-fabsf(h)));
    return (1.0f - smoothing) * (fmaxf(-h, 0.0f) + tail) + smoothing * (fmaxf(h, 0.0f) + tail);
}

// WARPS warps per pair, pairs blockIdx.x * (warps of the CTA / WARPS) + ...: both answers' sums, the pair's loss and the gradient at every logp of
// the two.  loss (may be null): the mean, where one CTA has all pairs.
constexpr int PAIR_THREADS = 256;
template <int WARPS>
__global__ void __launch_bounds__(PAIR_THREADS) pair_kernel(const PairParams P, float* loss) {
    pdl_enter();
    constexpr int ALL = PAIR_THREADS / 32, STEP = 32 * WARPS;
    __shared__ double part[ALL];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp % WARPS * 32 + lane;
    double total = 0.0;                                        // of this warp's pairs' losses
    for (int64_t i = (int64_t)blockIdx.x * (ALL / WARPS) + warp / WARPS; i < P.pairs; i += (int64_t)gridDim.x * (ALL / WARPS)) {
        const int64_t a = whole_at(P.offsets, P.off_wide, 2 * i), b = whole_at(P.offsets, P.off_wide, 2 * i + 1), e = whole_at(P.offsets, P.off_wide, 2 * i + 2);
        if (!(0 <= a && a <= b && b <= e && e <= P.rows)) {    // (the same for all warps of the pair)
            if (first == 0) { note(P.status, SRQ_ERR_INVALID_ARG); P.pair_loss[i] = 0.0f; }
            continue;
        }
        double s = 0.0;
#pragma unroll 4
        for (int64_t r = a + first; r < e; r += STEP) {
            const int64_t t = whole_at(P.targets, P.wide, r);
            const bool counts = t >= 0 && t < P.classes;
            const double d = counts ? (double)P.logp[r] - (double)P.ref[r] : 0.0;
            s += r < b ? d : -d;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        if constexpr (WARPS > 1) {
            if (lane == 0) part[warp] = s;
            __syncthreads();
            s = 0.0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += part[w];
            __syncthreads();
        }
        const float h = (float)(s * (double)P.beta), mine = pair_loss_of(h, P.smoothing);
        total += (double)mine;
        if (first == 0) {
            P.pair_loss[i] = mine;
            if (abs_word(h) >= 0x7F800000u) note(P.status, SRQ_ERR_NONFINITE);
        }
        const float c = (P.smoothing - 1.0f / (1.0f + expf(h))) * P.beta / (float)P.pairs;
        for (int64_t r = a + first; r < e; r += STEP) P.dlogp[r] = r < b ? c : -c;
    }
    if (loss) {
        __syncthreads();
        if (lane == 0) part[warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            double t = 0.0;
#pragma unroll
            for (int w = 0; w < ALL; ++w) t += part[w];
            loss[0] = (float)(t / (double)P.pairs);
        }
    }
}

// CTAs per row.  A CTA of 128 threads holds 32 KB of a row in shared memory (six CTAs per SM), one of 32 threads 8 KB, which is enough for short
// rows.  A gradient's rows (keep) are shared by as many CTAs as hold them, up to eight; all long rows where there are too few to fill the
// device.  Sums alone go through the row 32 KB at a time and share nothing (16 pairs of 256 on 50257 classes: sums with a cluster of four 180 us, one
// CTA 140; gradients by one CTA a row 257, by four 242).
static int row_parts(int64_t rows, int64_t vectors, bool keep) {
    const int sms = sm_count();
    int p = 1;
    while (p < 8 && ((keep && vectors > (int64_t)p * 128 * ROW_SLOTS) || (rows * p < 4 * (int64_t)sms && vectors >= 512 * (int64_t)p))) p <<= 1;
    return p;
}

template <typename T, int MODE, int NT>
static cudaError_t launch_rows_of(const RowParams& P, int64_t vectors, cudaStream_t st) {
    const int64_t each = ((vectors + P.parts - 1) / P.parts + NT - 1) / NT;
    if (P.rows * P.parts > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(P.rows * P.parts)); cfg.blockDim = dim3(NT); cfg.stream = st;
    cfg.dynamicSmemBytes = (size_t)(each < ROW_SLOTS ? each : ROW_SLOTS) * NT * 16;
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
    return cudaLaunchKernelEx(&cfg, row_kernel<T, MODE, NT>, P);
}
template <typename T, int MODE>
static cudaError_t launch_rows(RowParams P, cudaStream_t st) {
    // rows that do not begin at 16-byte boundaries have a vector more
    const int64_t bytes = P.classes * (int64_t)sizeof(T), vectors = bytes / 16 + (bytes % 16 || P.ld * (int64_t)sizeof(T) % 16 ? 2 : 0);
    P.parts = row_parts(P.rows, vectors, MODE != ROW_LOGP);
    return (vectors + P.parts - 1) / P.parts <= 32 * ROW_SLOTS ? launch_rows_of<T, MODE, 32>(P, vectors, st) : launch_rows_of<T, MODE, 128>(P, vectors, st);
}
template <int MODE>
static cudaError_t launch_rows(const RowParams& P, int32_t dt, cudaStream_t st) {
    return dt == SRQ_F32 ? launch_rows<float, MODE>(P, st) : launch_rows<__nv_bfloat16, MODE>(P, st);
}

static RowParams row_params(const LogitsArgs& a) {
    RowParams P = {};
    P.x = a.x; P.rows = a.rows; P.classes = a.classes; P.ld = a.ld;
    P.targets = a.targets; P.wide = a.target_t == SRQ_I64;
    const double k = 1.4426950408889634074 / (double)a.temperature;
    P.k = (float)k;
    while ((double)P.k >= k) P.k = nextafterf(P.k, 0.0f);      // what is lacking is positive: minus infinity times it is no NaN
    P.k_low = (float)(k - (double)P.k); P.inv_t = 1.0f / a.temperature; P.t = a.temperature;
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
    return launch_rows<ROW_LSE>(P, a.dt, st);
}
static cudaError_t launch_loss_sum(const float* x, int64_t n, double scale, float* out, cudaStream_t st) {
    count_launch();
    return launch_pdl(loss_sum_kernel, dim3(1), dim3(1024), 0, st, x, n, scale, out);
}
cudaError_t launch_policy(const LogitsArgs& a, const PolicyArgs& p, cudaStream_t st) {
    RowParams P = row_params(a);
    P.logp = p.logp; P.dx = p.dx; P.ldx = p.ldx; P.old = p.old; P.advantage = p.advantage; P.weight = p.weight;
    P.ref = p.h.kl_coef != 0.0f ? p.ref : nullptr;             // (0 times an exponential that left binary32 would be NaN)
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
    P.logp = p.logp; P.offsets = p.offsets; P.off_wide = p.offset_t == SRQ_I64; P.last = 2 * p.pairs; P.clear_rest = p.h.clear_rest;
    cudaError_t e = a.rows ? launch_rows<ROW_LOGP>(P, a.dt, st) : cudaSuccess;
    if (e != cudaSuccess) return e;
    PairParams Q = {};
    Q.logp = p.logp; Q.ref = p.ref; Q.targets = a.targets; Q.wide = P.wide; Q.offsets = p.offsets; Q.off_wide = P.off_wide;
    Q.rows = a.rows; Q.classes = a.classes; Q.pairs = p.pairs; Q.beta = p.h.beta; Q.smoothing = p.h.label_smoothing;
    Q.pair_loss = p.pair_loss; Q.dlogp = dlogp; Q.status = a.status;
    // a few short pairs: a warp each in one CTA, which then knows the mean (a launch less: two pairs of 40 tokens 17 -> 14 us)
    const bool one = p.pairs <= PAIR_THREADS / 32 && a.rows <= 4096;
    e = one ? launch_pdl(pair_kernel<1>, dim3(1), dim3(PAIR_THREADS), 0, st, Q, p.loss)
            : launch_pdl(pair_kernel<PAIR_THREADS / 32>, dim3((unsigned)p.pairs), dim3(PAIR_THREADS), 0, st, Q, (float*)nullptr);
    count_launch();
    if (e != cudaSuccess) return e;
    if (p.dx && a.rows) {
        P.dlogp = dlogp; P.dx = p.dx; P.ldx = p.ldx; P.logp = nullptr;
        e = launch_rows<ROW_GRAD>(P, a.dt, st);
        if (e != cudaSuccess) return e;
    }
    return p.loss && !one ? launch_loss_sum(p.pair_loss, p.pairs, 1.0 / (double)p.pairs, p.loss, st) : cudaSuccess;
}

}  // namespace srq
