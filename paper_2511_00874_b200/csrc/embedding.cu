// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Forward: a copy of rows; bound by HBM (rows that come up often are read from L2).  16384 tokens x 4096 bfloat16: 30.5 us, 5.8 TB/s.
//
// Gradient.  The tokens are sorted by id (stable, radix), so that the tokens of one row of the table are neighbours, in the order
// in which they came.  Most rows of a table have no token at all and are written as zeros, which is most of the traffic and needs no
// sorted tokens: while one cluster of CTAs sorts, all others look through the ids for those of their own rows and clear the rest.
// Then the sorted tokens are cut into equal pieces, one per CTA, however uneven the ids are.  A CTA writes the rows that begin and end in
// its piece; sums of a row that began in an earlier piece or goes on in the next one are kept aside as partial rows (binary32) and
// joined by a third kernel in the order of the pieces.  No atomics on sums: the result repeats bit for bit.
// 16384 tokens, a table of 32000 x 2048: 80 us (4.1 TB/s over all bytes), of it sorting and clearing 46, sums 23, joins 10; the three steps
// follow one another, which is what is left.  All rows by one merge of sorted tokens and row ends, after a sort in one CTA: 152 us.
#include "train.cuh"

namespace srq {

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------
struct EmbedFwdParams {
    const void* table; int64_t rows, cols, ld;
    const void* ids; int32_t wide; int64_t tokens; float scale;
    void* out; int64_t ld_out; uint32_t* status;
    int32_t lanes, log_lanes;                   // lanes per token (power of two up to 32)
    int64_t turns;                              // pieces of EMBED_U * lanes vectors a row is cut into
    int32_t narrow;                             // tokens * turns stays below 2^31
};
constexpr int EMBED_U = 4;                      // vectors in flight per lane

// N elements of a row as they lie in memory: one, or eight that are 16-byte aligned (one or two vectors).
template <typename T, int N> struct Raw;
template <typename T> struct Raw<T, 1> {
    T e;
    __device__ __forceinline__ void clear() { e = (T)0.0f; }
    __device__ __forceinline__ void load(const T* p) { e = *p; }
    __device__ __forceinline__ void values(float v[1]) const { v[0] = (float)e; }
};
template <> struct Raw<__nv_bfloat16, 8> {
    uint4 a;
    __device__ __forceinline__ void clear() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void values(float v[8]) const {
        v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
        v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
    }
};
template <> struct Raw<float, 8> {
    float4 a, b;
    __device__ __forceinline__ void clear() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void values(float v[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};

// VEC: eight elements of a row at a time, else one.
template <typename I, typename O, bool VEC>
__global__ void __launch_bounds__(256, 6) embedding_fwd_kernel(const EmbedFwdParams P) {
    pdl_enter();
    constexpr int N = VEC ? 8 : 1;
    const int lane = threadIdx.x & (P.lanes - 1);
    const int64_t w = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> P.log_lanes;
    // (a division in 64 bits takes more instructions than the copy)
    const int64_t token = P.narrow ? (int64_t)((uint32_t)w / (uint32_t)P.turns) : w / P.turns, turn = w - token * P.turns;
    if (token >= P.tokens) return;
    const int64_t id = whole_at(P.ids, P.wide, token);
    const bool valid = id >= 0 && id < P.rows;
    if (id >= P.rows && lane == 0 && turn == 0) note(P.status, SRQ_ERR_INVALID_ARG);
    const I* src = reinterpret_cast<const I*>(P.table) + (valid ? id : 0) * P.ld;
    O* dst = reinterpret_cast<O*>(P.out) + token * P.ld_out;
    const int64_t c0 = (turn * EMBED_U * P.lanes + lane) * N, step = (int64_t)P.lanes * N;
    Raw<I, N> raw[EMBED_U];
#pragma unroll
    for (int u = 0; u < EMBED_U; ++u) {
        raw[u].clear();
        if (valid && c0 + u * step < P.cols) raw[u].load(src + c0 + u * step);
    }
#pragma unroll
    for (int u = 0; u < EMBED_U; ++u) {
        const int64_t c = c0 + u * step;
        if (c >= P.cols) break;
        float v[N];
        raw[u].values(v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] *= P.scale;
        if constexpr (VEC) store8<O>(dst, c, P.cols, true, v);
        else dst[c] = (O)v[0];
    }
}

static bool whole_vectors(const void* p, int64_t ld, int64_t cols, int32_t dt) {
    return cols % 8 == 0 && ld % (dt == SRQ_F32 ? 4 : 8) == 0 && ((uintptr_t)p & 15u) == 0;
}

cudaError_t launch_embedding_fwd(const EmbedFwdArgs& a, cudaStream_t st) {
    EmbedFwdParams P;
    P.table = a.table; P.rows = a.rows; P.cols = a.cols; P.ld = a.ld; P.ids = a.ids; P.wide = a.id_t == SRQ_I64; P.tokens = a.tokens;
    P.scale = a.scale; P.out = a.out; P.ld_out = a.ld_out; P.status = a.status;
    const bool vec = whole_vectors(a.table, a.ld, a.cols, a.dt) && whole_vectors(a.out, a.ld_out, a.cols, a.out_dt);
    const int64_t n = vec ? a.cols / 8 : a.cols;               // vectors of a row
    P.log_lanes = 0;
    while (P.log_lanes < 5 && (1 << P.log_lanes) < n) ++P.log_lanes;
    P.lanes = 1 << P.log_lanes;
    P.turns = (n + (int64_t)EMBED_U * P.lanes - 1) / ((int64_t)EMBED_U * P.lanes);
    P.narrow = a.tokens * P.turns + 256 < 0x7FFFFFFFll;
    const int64_t ctas = (a.tokens * P.turns * P.lanes + 255) / 256;
    if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas), block(256);
    typedef __nv_bfloat16 H;
    const bool f = a.dt == SRQ_F32, of = a.out_dt == SRQ_F32;
    count_launch();
#define SRQ_EMBED(V) (f ? (of ? launch_pdl(embedding_fwd_kernel<float, float, V>, grid, block, 0, st, P) : launch_pdl(embedding_fwd_kernel<float, H, V>, grid, block, 0, st, P)) \
                        : (of ? launch_pdl(embedding_fwd_kernel<H, float, V>, grid, block, 0, st, P) : launch_pdl(embedding_fwd_kernel<H, H, V>, grid, block, 0, st, P)))
    return vec ? SRQ_EMBED(true) : SRQ_EMBED(false);
#undef SRQ_EMBED
}

// ------------------------------------------------------------------------------------------------
// sorting
// ------------------------------------------------------------------------------------------------
// Radix sort, lowest digits first (of at most 9 bits, where several CTAs take part).  Keys are ids; everything without a gradient has the key `rows`, which sorts last.
constexpr int SORT_BINS = 512, SORT_ONE = 65536, SORT_ONE_THREADS = 512, SORT_TILE = 4096, SORT_THREADS = 512, SORT_MAX_BLOCKS = 128;

struct SortPlan { int total, passes, bits; };
static SortPlan sort_plan(int64_t rows) {
    SortPlan p;
    p.total = 1;
    while (p.total < 31 && ((int64_t)1 << p.total) <= rows) ++p.total;  // keys 0 .. rows
    p.passes = (p.total + 8) / 9;
    p.bits = (p.total + p.passes - 1) / p.passes;
    return p;
}

__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t rows, uint32_t* status) {
    if (id >= rows) note(status, SRQ_ERR_INVALID_ARG);
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

// Ranks a warp's keys, 32 at a time in their order: place among the warp's keys of the same digit so far.  counts: the warp's own.
// Who has the same digit is found by a vote per bit.
__device__ __forceinline__ uint32_t rank_in_warp(uint32_t digit, int bits, bool active, uint16_t* counts, int lane) {
    uint32_t same = __ballot_sync(0xFFFFFFFFu, active);
    for (int b = 0; b < bits; ++b) {
        const uint32_t set = __ballot_sync(0xFFFFFFFFu, (digit >> b) & 1u);
        same &= (digit >> b) & 1u ? set : ~set;
    }
    uint32_t rank = 0;
    const uint32_t before = same & ((1u << lane) - 1u);
    if (active) rank = counts[digit] + __popc(before);
    __syncwarp();
    if (active && before == 0) counts[digit] = (uint16_t)(counts[digit] + __popc(same));
    __syncwarp();
    return rank;
}

// Exclusive sums over the bins (one per thread of the first `bins`); every thread of the CTA takes part.
template <int THREADS>
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t x, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t s = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    uint32_t before = lane < warp ? warp_sums[lane] : 0;       // at most 32 warps
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
    __syncthreads();
    return before + s - x;
}

// All passes in one launch, for up to SORT_ONE tokens, by one CTA or a cluster of eight, the first of the grid; the others clear the rows
// without a token.  CTA q holds places q * per .. (q + 1) * per - 1 in shared memory.  A thread has neighbouring tokens and a counter of its own
// for each value of a digit, so that a token's rank is one addition; the counters' exclusive sums, digit by digit and thread by
// thread, with the other CTAs' totals before them, are the places, and the tokens go there through distributed shared memory.
// 16384 tokens, ids below 32000: 52 us with one CTA alone (its shared memory is the bound).
constexpr int ONE_BITS = 6, ONE_BINS = 1 << ONE_BITS, ONE_PER = SORT_ONE / 8, ONE_MOST = ONE_PER / SORT_ONE_THREADS + 1;
struct SortOneShared {                          // then uint32_t key[per], uint16_t place[per]
    uint4 count[ONE_BINS * SORT_ONE_THREADS / 8];              // 16-bit counters [digit][thread], eight to a unit
    uint32_t totals[8][ONE_BINS], start[ONE_BINS], base[ONE_BINS];
    uint32_t sums[32];
};
// Where unit u of the counters lies: threads that read eight units in a row each would meet in the same banks otherwise.
__device__ __forceinline__ int unit_at(int u) { return (u & ~7) | ((u + (u >> 3)) & 7); }
__device__ __forceinline__ uint16_t& counter(SortOneShared& S, uint32_t digit, int tid) {
    const int e = (int)digit * SORT_ONE_THREADS + tid;
    return reinterpret_cast<uint16_t*>(&S.count[unit_at(e >> 3)])[e & 7];
}
__device__ __forceinline__ uint32_t in_cta(const void* p, uint32_t cta) {      // the same shared variable of another CTA of the cluster
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    return a;
}
__device__ __forceinline__ void cluster_barrier(int parts) {
    __syncwarp();                                              // the cluster's barrier takes converged warps
    if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
}
struct SortOneParams {
    const void* ids; int32_t wide; int32_t n; int64_t rows; int32_t bits, parts, log_per;
    uint32_t* keys; uint32_t* perm; uint32_t* status;
    char* out; int64_t pitch, bytes;            // rows to clear: distance and length in bytes
};

// Rows of this CTA's share that no token has become zero.  flags: shared memory, a byte per row.
constexpr int CLEAR_ROWS = ONE_BINS * SORT_ONE_THREADS * 2;    // at a time: the memory of the counters
__device__ __forceinline__ void clear_rows(const SortOneParams& P, uint8_t* flags) {
    const int tid = threadIdx.x;
    const int64_t share = blockIdx.x - P.parts, shares = gridDim.x - P.parts;
    const int64_t a = P.rows / shares * share + P.rows % shares * share / shares, b = P.rows / shares * (share + 1) + P.rows % shares * (share + 1) / shares;
    const uintptr_t odd = (uintptr_t)P.out | (uintptr_t)P.pitch | (uintptr_t)P.bytes;
    const bool vec = (odd & 31u) == 0;
    Word8 zero;
#pragma unroll
    for (int q = 0; q < 8; ++q) zero.w[q] = 0;
    for (int64_t r0 = a; r0 < b; r0 += CLEAR_ROWS) {
        const int rows = (int)(b - r0 < CLEAR_ROWS ? b - r0 : CLEAR_ROWS);
        __syncthreads();
        for (int r = tid; r < rows; r += SORT_ONE_THREADS) flags[r] = 0;
        __syncthreads();
        constexpr int AHEAD = 16;
        for (int i = tid; i < P.n; i += AHEAD * SORT_ONE_THREADS) {
            int64_t id[AHEAD];
#pragma unroll
            for (int t = 0; t < AHEAD; ++t) id[t] = i + t * SORT_ONE_THREADS < P.n ? whole_at(P.ids, P.wide, i + t * SORT_ONE_THREADS) : -1;
#pragma unroll
            for (int t = 0; t < AHEAD; ++t)
                if (id[t] >= r0 && id[t] < r0 + rows) flags[id[t] - r0] = 1;
        }
        __syncthreads();
        for (int r = tid >> 5; r < rows; r += SORT_ONE_THREADS / 32) {
            if (flags[r]) continue;
            char* p = P.out + (r0 + r) * P.pitch;
            if (vec) {
                for (int c = (tid & 31) * 32; c < (int)P.bytes; c += 1024) store32(p + c, zero);
            } else {
                for (int c = (tid & 31) * 2; c < (int)P.bytes; c += 64) *reinterpret_cast<uint16_t*>(p + c) = 0;
            }
        }
    }
}

__global__ void __launch_bounds__(SORT_ONE_THREADS, 2) sort_one_kernel(const SortOneParams P) {
    pdl_enter();
    extern __shared__ uint4 raw[];
    if ((int)blockIdx.x >= P.parts) {                          // (whole clusters)
        clear_rows(P, reinterpret_cast<uint8_t*>(raw));
        return;
    }
    SortOneShared& S = *reinterpret_cast<SortOneShared*>(raw);
    const int tid = threadIdx.x, rank = blockIdx.x, per = 1 << P.log_per;
    uint32_t* S_key = reinterpret_cast<uint32_t*>(&S + 1);
    uint16_t* S_place = reinterpret_cast<uint16_t*>(S_key + per);
    const int rest = P.n - rank * per, n = rest < 0 ? 0 : rest < per ? rest : per;
    // an odd number of tokens per thread: neighbouring threads' tokens lie in different banks
    const int each = ((n + SORT_ONE_THREADS - 1) / SORT_ONE_THREADS) | 1, first = tid * each;
    {
        int64_t id[ONE_MOST];                                  // all loads first: one wait
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            const int i = t * SORT_ONE_THREADS + tid;
            id[t] = i < n ? whole_at(P.ids, P.wide, (int64_t)rank * per + i) : -1;
        }
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            const int i = t * SORT_ONE_THREADS + tid;
            if (i < n) { S_key[i] = key_of(id[t], P.rows, P.status); S_place[i] = (uint16_t)(rank * per + i); }
        }
    }
    cluster_barrier(P.parts);                                  // every CTA of the cluster is there
    for (int shift = 0; shift < P.bits; shift += ONE_BITS) {
        for (int u = tid; u < ONE_BINS * SORT_ONE_THREADS / 8; u += SORT_ONE_THREADS) S.count[u] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        uint32_t key[ONE_MOST], own[ONE_MOST];                 // own: the token in the upper half, its rank among the thread's
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            if (t >= each || first + t >= n) break;
            key[t] = S_key[first + t];
            uint16_t& c = counter(S, (key[t] >> shift) & (ONE_BINS - 1), tid);
            own[t] = (uint32_t)S_place[first + t] << 16 | c;
            c = (uint16_t)(c + 1);
        }
        __syncthreads();
        // exclusive sums over this CTA's counters; a thread has ONE_BINS of them in a row, all of one digit
        uint4 w[ONE_BINS / 8];
        uint32_t total = 0;
#pragma unroll
        for (int q = 0; q < ONE_BINS / 8; ++q) {
            w[q] = S.count[unit_at(tid * (ONE_BINS / 8) + q)];
            const uint32_t pairs = w[q].x + w[q].y + w[q].z + w[q].w;           // two 16-bit sums: at most 8 * 17 each
            total += (pairs & 0xFFFFu) + (pairs >> 16);
        }
        uint32_t at = exclusive_scan<SORT_ONE_THREADS>(total, S.sums);
        constexpr int PER_DIGIT = SORT_ONE_THREADS / ONE_BINS;                 // threads whose counters are one digit's
        if (tid % PER_DIGIT == 0) S.start[tid / PER_DIGIT] = at;
#pragma unroll
        for (int q = 0; q < ONE_BINS / 8; ++q) {
            uint32_t* x = reinterpret_cast<uint32_t*>(&w[q]);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint32_t lo = x[h] & 0xFFFFu, hi = x[h] >> 16;
                x[h] = at | (at + lo) << 16;
                at += lo + hi;
            }
            S.count[unit_at(tid * (ONE_BINS / 8) + q)] = w[q];
        }
        __syncthreads();
        if (tid < ONE_BINS) {                                  // this CTA's totals, to every CTA
            const uint32_t mine = (tid + 1 < ONE_BINS ? S.start[tid + 1] : (uint32_t)n) - S.start[tid];
            for (int q = 0; q < P.parts; ++q)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(&S.totals[rank][tid], q)), "r"(mine) : "memory");
        }
        cluster_barrier(P.parts);
        if (tid < 32) {                                        // two digits per lane: tokens of smaller digits, and of these in the CTAs before
            uint32_t all[2] = {0, 0}, before[2] = {0, 0};
            for (int q = 0; q < P.parts; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t c = S.totals[q][2 * tid + h];
                    all[h] += c;
                    if (q < rank) before[h] += c;
                }
            uint32_t s = all[0] + all[1];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, s, d);
                if (tid >= d) s += o;
            }
            s -= all[0] + all[1];
            S.base[2 * tid] = s + before[0] - S.start[2 * tid];
            S.base[2 * tid + 1] = s + all[0] + before[1] - S.start[2 * tid + 1];
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            if (t >= each || first + t >= n) break;
            const uint32_t d = (key[t] >> shift) & (ONE_BINS - 1), to = S.base[d] + counter(S, d, tid) + (own[t] & 0xFFFFu);
            const uint32_t cta = to >> P.log_per, i = to & (uint32_t)(per - 1);
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(&S_key[i], cta)), "r"(key[t]) : "memory");
            asm volatile("st.shared::cluster.u16 [%0], %1;" ::"r"(in_cta(&S_place[i], cta)), "h"((uint16_t)(own[t] >> 16)) : "memory");
        }
        cluster_barrier(P.parts);
    }
    for (int i = tid; i < n; i += SORT_ONE_THREADS) { P.keys[rank * per + i] = S_key[i]; P.perm[rank * per + i] = S_place[i]; }
}

// One pass over many CTAs: a CTA takes `per` neighbouring tokens (a multiple of SORT_TILE).  ids != nullptr: the first pass.
struct SortParams {
    const void* ids; int32_t wide; int64_t n, rows; int64_t per; int32_t shift, bits;
    const uint32_t* key_in; const uint32_t* place_in; uint32_t* key_out; uint32_t* place_out;
    uint32_t* hist;                             // [blocks][SORT_BINS]
    uint32_t* status;
};
__global__ void __launch_bounds__(SORT_THREADS) sort_count_kernel(const SortParams P) {
    pdl_enter();
    __shared__ uint32_t count[SORT_BINS];
    const int tid = threadIdx.x;
    count[tid] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * P.per, end = first + P.per < P.n ? first + P.per : P.n;
    const uint32_t mask = (1u << P.bits) - 1u;
    for (int64_t tile = first; tile < end; tile += SORT_TILE) {
        int64_t id[SORT_TILE / SORT_THREADS];
#pragma unroll
        for (int t = 0; t < SORT_TILE / SORT_THREADS; ++t) {
            const int64_t i = tile + t * SORT_THREADS + tid;
            id[t] = i >= end ? -1 : P.ids ? whole_at(P.ids, P.wide, i) : (int64_t)P.key_in[i];
        }
#pragma unroll
        for (int t = 0; t < SORT_TILE / SORT_THREADS; ++t) {
            if (tile + t * SORT_THREADS + tid >= end) continue;
            const uint32_t k = P.ids ? key_of(id[t], P.rows, P.status) : (uint32_t)id[t];
            atomicAdd(&count[(k >> P.shift) & mask], 1u);
        }
    }
    __syncthreads();
    P.hist[(int64_t)blockIdx.x * SORT_BINS + tid] = count[tid];
}
__global__ void __launch_bounds__(SORT_THREADS) sort_scatter_kernel(const SortParams P) {
    pdl_enter();
    constexpr int WARPS = SORT_THREADS / 32, TURNS = SORT_TILE / SORT_THREADS;
    __shared__ uint16_t count[WARPS][SORT_BINS];
    __shared__ uint32_t base[SORT_BINS], sums[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t mine = 0, total = 0;                              // bin tid: tokens of it in the CTAs before, in all
#pragma unroll 8
    for (int b = 0; b < (int)gridDim.x; ++b) {
        const uint32_t c = P.hist[(int64_t)b * SORT_BINS + tid];
        if (b < (int)blockIdx.x) mine += c;
        total += c;
    }
    base[tid] = exclusive_scan<SORT_THREADS>(total, sums) + mine;
    const int64_t first = blockIdx.x * P.per, end = first + P.per < P.n ? first + P.per : P.n;
    const uint32_t mask = (1u << P.bits) - 1u;
    for (int64_t tile = first; tile < end; tile += SORT_TILE) {
        uint32_t key[TURNS], rank[TURNS];
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t i = tile + (warp * TURNS + t) * 32 + lane;
            key[t] = i >= end ? 0u : P.ids ? key_of(whole_at(P.ids, P.wide, i), P.rows, nullptr) : P.key_in[i];
        }
        for (int i = tid; i < WARPS * SORT_BINS / 2; i += SORT_THREADS) reinterpret_cast<uint32_t*>(&count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const bool active = tile + (warp * TURNS + t) * 32 + lane < end;
            rank[t] = rank_in_warp((key[t] >> P.shift) & mask, P.bits, active, count[warp], lane);
        }
        __syncthreads();
        uint32_t here = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { const uint32_t c = count[w][tid]; count[w][tid] = (uint16_t)here; here += c; }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t i = tile + (warp * TURNS + t) * 32 + lane;
            if (i < end) {
                const uint32_t d = (key[t] >> P.shift) & mask, to = base[d] + count[warp][d] + rank[t];
                P.key_out[to] = key[t];
                P.place_out[to] = P.ids ? (uint32_t)i : P.place_in[i];
            }
        }
        __syncthreads();
        base[tid] += here;
    }
}

// ------------------------------------------------------------------------------------------------
// rows
// ------------------------------------------------------------------------------------------------
constexpr int ROWS_THREADS = 256;

struct alignas(8) PieceInfo { uint32_t row; uint16_t opened, closed; };     // first row of the piece; begun in an earlier piece; ends in this one

struct EmbedBwdParams {
    const uint32_t* keys; const uint32_t* perm; int64_t tokens, rows, cols;
    const void* dout; int64_t ld; void* out; int64_t ld_out; float scale;
    int32_t accumulate;
    int64_t pieces;
    PieceInfo* info; float* carry; float* head; int64_t ld_part;   // partial rows [pieces, ld_part]: at the end, at the beginning
};

template <typename T, int N>
__device__ __forceinline__ void load_cols(const T* row, int64_t c, float v[N]) {
    if constexpr (N == 8) load8<T>(row, c, c + 8, true, v);
    else v[0] = (float)row[c];
}
template <typename T, int N>
__device__ __forceinline__ void store_cols(T* row, int64_t c, const float v[N]) {
    if constexpr (N == 8) store8<T>(row, c, c + 8, true, v);
    else row[c] = (T)v[0];
}

// N columns per thread (8: whole aligned vectors), a slab of blockDim * N columns per CTA (blockIdx.y).
template <typename T, typename O, int N>
__global__ void __launch_bounds__(ROWS_THREADS, 4) embedding_rows_kernel(const EmbedBwdParams P) {
    pdl_enter();
    constexpr int BATCH = sizeof(T) == 4 && N == 8 ? 4 : 8;    // tokens whose rows are on their way together
    __shared__ uint32_t skey[ROWS_THREADS], sperm[ROWS_THREADS];
    const int tid = threadIdx.x;
    const int64_t piece = blockIdx.x, each = P.tokens / P.pieces, more = P.tokens % P.pieces;
    const int64_t j0 = each * piece + (more < piece ? more : piece), j1 = j0 + each + (piece < more ? 1 : 0);      // at least one token
    const uint32_t rows = (uint32_t)P.rows;
    const uint32_t r0 = P.keys[j0], before = j0 > 0 ? P.keys[j0 - 1] : ~0u, last = P.keys[j1 - 1], after = j1 < P.tokens ? P.keys[j1] : ~0u;
    const bool opened = before == r0 && r0 < rows, goes_on = after == last && last < rows;     // the first row has begun, the last one goes on
    if (tid == 0 && blockIdx.y == 0) P.info[piece] = PieceInfo{r0, (uint16_t)opened, (uint16_t)(r0 < rows && !(goes_on && last == r0))};
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + tid) * N;
    const bool mine = c < P.cols;                              // N == 8: whole vectors
    const T* x = reinterpret_cast<const T*>(P.dout) + c;
    O* out = reinterpret_cast<O*>(P.out) + c;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.0f;
    uint32_t row = r0;                                         // the row being added up
    const auto close = [&]() {                                 // it ends here
        if (mine) {
            if (row == r0 && opened) {
                store_cols<float, N>(P.head + piece * P.ld_part, c, acc);
            } else {
                float v[N];
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = acc[e] * P.scale;
                if (P.accumulate) {
                    float o[N];
                    load_cols<O, N>(out + row * P.ld_out, 0, o);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] += o[e];
                }
                store_cols<O, N>(out + row * P.ld_out, 0, v);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.0f;
    };
    for (int64_t base = j0; base < j1; base += blockDim.x) {
        const int here = (int)(j1 - base < (int64_t)blockDim.x ? j1 - base : (int64_t)blockDim.x);
        __syncthreads();
        if (tid < here) { skey[tid] = P.keys[base + tid]; sperm[tid] = P.perm[base + tid]; }
        __syncthreads();
        for (int t = 0; t < here; t += BATCH) {
            Raw<T, N> raw[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                raw[b].clear();
                if (t + b < here && mine && skey[t + b] < rows) raw[b].load(x + sperm[t + b] * P.ld);
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (t + b >= here) break;
                const uint32_t key = skey[t + b];
                if (key >= rows) break;                        // what has no gradient sorts last
                if (key != row) { close(); row = key; }
                float v[N];
                raw[b].values(v);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += v[e];
            }
        }
    }
    if (row >= rows) return;                                   // no token of the piece has a gradient
    if (!goes_on) close();
    else if (mine) store_cols<float, N>(P.carry + piece * P.ld_part, c, acc);
}

// Rows that span pieces: the pieces' partial rows, joined where the row ends.  A warp takes a piece and adds up the row that ends there, if it
// spans few; rows of more than JOIN_ALONE pieces are added up by all warps of the CTA together, one row after the other: warp g the partial
// rows g, g + JOIN_GROUPS, ..., then the warps' sums in order.
constexpr int JOIN_GROUPS = 8, JOIN_COLS = 32, JOIN_ALONE = 16;        // (threads: JOIN_GROUPS * JOIN_COLS, N columns each)
template <typename O, int N>
__global__ void __launch_bounds__(JOIN_GROUPS * JOIN_COLS) embedding_join_kernel(const EmbedBwdParams P) {
    pdl_enter();
    __shared__ int64_t first_of[JOIN_GROUPS];                  // of rows that are joined by all; -1: none
    __shared__ float sums[JOIN_GROUPS][JOIN_COLS * N];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t c = ((int64_t)blockIdx.y * JOIN_COLS + lane) * N;
    const bool mine = c < P.cols;
    const int64_t piece = (int64_t)blockIdx.x * JOIN_GROUPS + group;
    int64_t first = -1;
    PieceInfo me = {};
    if (piece < P.pieces) me = P.info[piece];
    if (me.opened && me.closed) {
        // where the row begins: the last piece before this one that did not find it open.  Those between hold nothing else.
        // 128 pieces are looked at together.
        bool found = false;
        for (first = piece - 1; !found;) {
            PieceInfo p[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                p[q] = PieceInfo{};
                if (first - 32 * q - lane > 0) p[q] = P.info[first - 32 * q - lane];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (found) break;
                const uint32_t who = __ballot_sync(0xFFFFFFFFu, !(p[q].row == me.row && p[q].opened));
                found = who != 0;
                first -= found ? __ffs(who) - 1 : 32;
            }
        }
    }
    // partial rows start, start + step, ... of the row that begins in piece `from` and ends in piece `to`, where its part is a head
    const auto add_up = [&](int64_t from, int64_t to, int start, int step, float acc[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.0f;
        if (!mine) return;
#pragma unroll 8
        for (int64_t p = from + start; p <= to; p += step) {
            float v[N];
            load_cols<float, N>((p < to ? P.carry : P.head) + p * P.ld_part, c, v);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += v[e];
        }
    };
    const auto finish = [&](uint32_t row, float acc[N]) {
        if (!mine) return;
        O* o = reinterpret_cast<O*>(P.out) + (int64_t)row * P.ld_out;
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] *= P.scale;
        if (P.accumulate) {
            load_cols<O, N>(o, c, v);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += v[e];
        }
        store_cols<O, N>(o, c, acc);
    };
    float acc[N];
    if (first >= 0 && piece - first < JOIN_ALONE) {
        add_up(first, piece, 0, 1, acc);
        finish(me.row, acc);
        first = -1;
    }
    if (lane == 0) first_of[group] = first;
    __syncthreads();
    for (int k = 0; k < JOIN_GROUPS; ++k) {
        if (first_of[k] < 0) continue;                         // the same for the whole CTA
        const int64_t last = (int64_t)blockIdx.x * JOIN_GROUPS + k;
        add_up(first_of[k], last, group, JOIN_GROUPS, acc);
#pragma unroll
        for (int e = 0; e < N; ++e) sums[group][lane * N + e] = acc[e];
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                acc[e] = 0.0f;
#pragma unroll
                for (int g = 0; g < JOIN_GROUPS; ++g) acc[e] += sums[g][lane * N + e];
            }
            finish(P.info[last].row, acc);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------
// workspace and launch
// ------------------------------------------------------------------------------------------------
// Pieces: enough for every SM to hold its share of CTAs, at least four tokens each.  The bound does not ask the device, since the
// workspace's size is the same for every one.
constexpr int64_t MAX_PIECES = 1184;
static int64_t piece_count(int64_t tokens) {
    const int64_t n = (tokens + 3) / 4;
    return n < 1 ? 1 : n < MAX_PIECES ? n : MAX_PIECES;
}
static int64_t part_pitch(int64_t cols) { return (cols + 63) / 64 * 64; }
struct EmbedScratch { uint32_t* key[2]; uint32_t* place[2]; uint32_t* hist; PieceInfo* info; float* carry; float* head; size_t bytes; };
static EmbedScratch embed_scratch(void* ws, int64_t tokens, int64_t cols) {
    EmbedScratch s;
    char* p = (char*)ws;
    size_t at = 0;
    auto take = [&](size_t n) { char* q = p + at; at += align_up(n); return q; };
    const int sets = tokens <= SORT_ONE ? 1 : 2;
    for (int i = 0; i < 2; ++i) {
        s.key[i] = i < sets ? (uint32_t*)take((size_t)tokens * 4) : nullptr;
        s.place[i] = i < sets ? (uint32_t*)take((size_t)tokens * 4) : nullptr;
    }
    s.hist = sets == 2 ? (uint32_t*)take((size_t)SORT_MAX_BLOCKS * SORT_BINS * 4) : nullptr;
    const int64_t pieces = piece_count(tokens);
    s.info = (PieceInfo*)take((size_t)pieces * sizeof(PieceInfo));
    s.carry = (float*)take((size_t)pieces * part_pitch(cols) * 4);
    s.head = (float*)take((size_t)pieces * part_pitch(cols) * 4);
    s.bytes = at;
    return s;
}
size_t embedding_bytes(int64_t tokens, int64_t cols) { return embed_scratch(nullptr, tokens, cols).bytes; }

template <typename T, typename O>
static cudaError_t launch_rows(const EmbedBwdParams& P, bool vec, cudaStream_t st) {
    const int64_t n = vec ? P.cols / 8 : P.cols;
    const int threads = n >= ROWS_THREADS ? ROWS_THREADS : (int)((n + 31) / 32 * 32);
    const dim3 grid((unsigned)P.pieces, (unsigned)((n + threads - 1) / threads)), block(threads);
    count_launch();
    cudaError_t e = vec ? launch_pdl(embedding_rows_kernel<T, O, 8>, grid, block, 0, st, P) : launch_pdl(embedding_rows_kernel<T, O, 1>, grid, block, 0, st, P);
    if (e != cudaSuccess || P.pieces == 1) return e;
    count_launch();
    const dim3 join((unsigned)((P.pieces + JOIN_GROUPS - 1) / JOIN_GROUPS), (unsigned)((n + JOIN_COLS - 1) / JOIN_COLS)), threads_of(JOIN_GROUPS * JOIN_COLS);
    return vec ? launch_pdl(embedding_join_kernel<O, 8>, join, threads_of, 0, st, P) : launch_pdl(embedding_join_kernel<O, 1>, join, threads_of, 0, st, P);
}

cudaError_t launch_embedding_bwd(const EmbedBwdArgs& a, cudaStream_t st) {
    const size_t esize = a.out_dt == SRQ_F32 ? 4 : 2;
    const auto clear_all = [&]() { return cudaMemset2DAsync(a.out, (size_t)a.ld_out * esize, 0, (size_t)a.cols * esize, (size_t)a.rows, st); };
    if (a.tokens == 0) return a.accumulate ? cudaSuccess : clear_all();
    const EmbedScratch s = embed_scratch(a.ws, a.tokens, a.cols);
    const SortPlan plan = sort_plan(a.rows);
    const int sms = sm_count();
    if (sms == 0) return cudaErrorUnknown;
    const int wide = a.id_t == SRQ_I64;
    int last = 0;                                              // buffers that hold the sorted tokens
    if (a.tokens <= SORT_ONE) {
        SortOneParams Q = {a.ids, wide, (int)a.tokens, a.rows, plan.total, 1, 0, s.key[0], s.place[0], a.status,
                           (char*)a.out, a.ld_out * (int64_t)esize, a.cols * (int64_t)esize};
        // one CTA for what its threads hold in four tokens each (a cluster's barriers cost more than they save), else eight
        Q.parts = a.tokens <= 4 * SORT_ONE_THREADS ? 1 : 8;
        while ((int64_t)Q.parts << Q.log_per < a.tokens) ++Q.log_per;
        const size_t smem = sizeof(SortOneShared) + ((size_t)6 << Q.log_per);
        cudaError_t e = cudaFuncSetAttribute(sort_one_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(SortOneShared) + 6 * ONE_PER));
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        // as many CTAs as the SMs have room for (113 KB each for two); where it accumulates there is nothing to clear
        const int resident = (smem <= 112 * 1024 ? 2 : 1) * sms / Q.parts * Q.parts;
        cfg.gridDim = dim3(a.accumulate ? Q.parts : resident > Q.parts ? resident : 2 * Q.parts); cfg.blockDim = dim3(SORT_ONE_THREADS);
        cfg.dynamicSmemBytes = smem; cfg.stream = st;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)Q.parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at; cfg.numAttrs = pdl_allowed(st) ? 2 : 1;
        count_launch();
        e = cudaLaunchKernelEx(&cfg, sort_one_kernel, Q);
        if (e != cudaSuccess) return e;
    } else {
        if (!a.accumulate) {                                   // here the ids are too many to be looked through by every CTA
            const cudaError_t e = clear_all();
            if (e != cudaSuccess) return e;
        }
        SortParams Q = {};
        Q.wide = wide; Q.n = a.tokens; Q.rows = a.rows; Q.bits = plan.bits; Q.hist = s.hist; Q.status = a.status;
        Q.per = (a.tokens + SORT_MAX_BLOCKS - 1) / SORT_MAX_BLOCKS;
        Q.per = (Q.per + SORT_TILE - 1) / SORT_TILE * SORT_TILE;
        const dim3 grid((unsigned)((a.tokens + Q.per - 1) / Q.per));
        for (int pass = 0; pass < plan.passes; ++pass) {
            Q.ids = pass == 0 ? a.ids : nullptr;
            Q.shift = pass * plan.bits;
            last = pass & 1;
            Q.key_in = s.key[1 - last]; Q.place_in = s.place[1 - last]; Q.key_out = s.key[last]; Q.place_out = s.place[last];
            count_launch();
            cudaError_t e = launch_pdl(sort_count_kernel, grid, dim3(SORT_THREADS), 0, st, Q);
            if (e != cudaSuccess) return e;
            count_launch();
            e = launch_pdl(sort_scatter_kernel, grid, dim3(SORT_THREADS), 0, st, Q);
            if (e != cudaSuccess) return e;
        }
    }
    EmbedBwdParams P;
    P.keys = s.key[last]; P.perm = s.place[last]; P.tokens = a.tokens; P.rows = a.rows; P.cols = a.cols;
    P.dout = a.dout; P.ld = a.ld; P.out = a.out; P.ld_out = a.ld_out; P.scale = a.scale; P.accumulate = a.accumulate;
    P.pieces = piece_count(a.tokens);
    P.info = s.info; P.carry = s.carry; P.head = s.head; P.ld_part = part_pitch(a.cols);
    const bool vec = whole_vectors(a.dout, a.ld, a.cols, a.dt) && whole_vectors(a.out, a.ld_out, a.cols, a.out_dt);
    typedef __nv_bfloat16 H;
    if (a.dt == SRQ_F32) return a.out_dt == SRQ_F32 ? launch_rows<float, float>(P, vec, st) : launch_rows<float, H>(P, vec, st);
    return a.out_dt == SRQ_F32 ? launch_rows<H, float>(P, vec, st) : launch_rows<H, H>(P, vec, st);
}

}  // namespace srq
