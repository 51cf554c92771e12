// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Forward: a copy of rows; bound by HBM (rows that come up often are read from L2).
//
// Gradient.  The tokens are sorted by id (stable, radix), so that the tokens of one row of the table are neighbours, in the order
// in which they came.  The rows of the table and the sorted tokens are then merged into one list (a row's tokens, then the row's end)
// and cut into equal pieces, one per CTA: the merge path of sparse products (Merrill and Garland, SC'16), which gives
// every CTA the same number of rows to write and tokens to add, however uneven the ids are.  Item j of the sorted tokens stands
// at place j + id_j of the list, so that a cut is found by one search (in shared memory, where the sort ends there).  A CTA writes the rows that end in its piece, zero rows
// included, once each; sums of a row that began in an earlier piece or goes on in the next one are kept aside as
// partial rows (binary32) and joined by a second kernel in the order of the pieces.  No atomics: the result repeats bit for bit.
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
    const int64_t token = w / P.turns, turn = w - token * P.turns;
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
constexpr int SORT_BINS = 512, SORT_ONE = 16384, SORT_ONE_THREADS = 1024, SORT_TILE = 4096, SORT_THREADS = 512, SORT_MAX_BLOCKS = 128;

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

// Tokens before place d of the merged list: the first j with j + key_j >= d (one thread).
__device__ __forceinline__ int64_t tokens_before(const uint32_t* keys, int64_t n, int64_t d) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (mid + (int64_t)keys[mid] < d) lo = mid + 1; else hi = mid;
    }
    return lo;
}
// Where piece p begins in a list of `items`.
__device__ __forceinline__ int64_t piece_begin(int64_t items, int64_t pieces, int64_t p) { return items / pieces * p + (items % pieces) * p / pieces; }

// All passes in one CTA, for up to SORT_ONE tokens, and the pieces' first tokens (cuts; null: not wanted).  A thread has neighbouring tokens and
// a counter of its own for each value of a digit, so that a token's rank is one addition; the counters' exclusive sums, digit
// by digit and thread by thread, are the places.  (Ranking 32 tokens at a time by the warp's votes took 34 us for 16384 tokens.)
constexpr int ONE_BITS = 5, ONE_BINS = 1 << ONE_BITS, ONE_MOST = SORT_ONE / SORT_ONE_THREADS;
struct SortOneShared {
    uint32_t key[SORT_ONE];
    uint16_t place[SORT_ONE];
    uint16_t count[ONE_BINS][SORT_ONE_THREADS];
    uint32_t sums[32];
};
__global__ void __launch_bounds__(SORT_ONE_THREADS) sort_one_kernel(const void* ids, int wide, int n, int64_t rows, int bits, uint32_t* keys, uint32_t* perm,
                                                                    int64_t* cuts, int64_t pieces, uint32_t* status) {
    pdl_enter();
    extern __shared__ char raw[];
    SortOneShared& S = *reinterpret_cast<SortOneShared*>(raw);
    const int tid = threadIdx.x, each = (n + SORT_ONE_THREADS - 1) / SORT_ONE_THREADS, first = tid * each;
    {
        int64_t id[ONE_MOST];                                  // all loads first: one wait instead of sixteen
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) id[t] = t * SORT_ONE_THREADS + tid < n ? whole_at(ids, wide, t * SORT_ONE_THREADS + tid) : -1;
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            const int i = t * SORT_ONE_THREADS + tid;
            if (i < n) { S.key[i] = key_of(id[t], rows, status); S.place[i] = (uint16_t)i; }
        }
    }
    for (int shift = 0; shift < bits; shift += ONE_BITS) {
        uint4* mine = reinterpret_cast<uint4*>(&S.count[0][0]) + tid * 4;      // 32 counters in the order of the sums: 64 bytes
#pragma unroll
        for (int q = 0; q < 4; ++q) mine[q] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        uint32_t key[ONE_MOST], rank[ONE_MOST];                // rank: the token in the upper half
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            if (t >= each || first + t >= n) break;
            key[t] = S.key[first + t];
            uint16_t& c = S.count[(key[t] >> shift) & (ONE_BINS - 1)][tid];
            rank[t] = (uint32_t)S.place[first + t] << 16 | c;
            c = (uint16_t)(c + 1);
        }
        __syncthreads();
        uint32_t w[16], total = 0;                             // pairs of counters
#pragma unroll
        for (int q = 0; q < 4; ++q) { const uint4 x = mine[q]; w[4 * q] = x.x; w[4 * q + 1] = x.y; w[4 * q + 2] = x.z; w[4 * q + 3] = x.w; }
#pragma unroll
        for (int q = 0; q < 16; ++q) total += (w[q] & 0xFFFFu) + (w[q] >> 16);
        uint32_t at = exclusive_scan<SORT_ONE_THREADS>(total, S.sums);
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint32_t lo = w[q] & 0xFFFFu, hi = w[q] >> 16;
            w[q] = at | (at + lo) << 16;
            at += lo + hi;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) mine[q] = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < ONE_MOST; ++t) {
            if (t >= each || first + t >= n) break;
            const uint32_t to = S.count[(key[t] >> shift) & (ONE_BINS - 1)][tid] + (rank[t] & 0xFFFFu);
            S.key[to] = key[t];
            S.place[to] = (uint16_t)(rank[t] >> 16);
        }
        __syncthreads();
    }
    for (int i = tid; i < n; i += SORT_ONE_THREADS) { keys[i] = S.key[i]; perm[i] = S.place[i]; }
    if (cuts)
        for (int64_t p = tid; p <= pieces; p += SORT_ONE_THREADS) cuts[p] = tokens_before(S.key, n, piece_begin(rows + n, pieces, p));
}
// The same for tokens that are sorted already.
__global__ void __launch_bounds__(256) cut_kernel(const uint32_t* keys, int64_t n, int64_t rows, int64_t* cuts, int64_t pieces) {
    pdl_enter();
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p <= pieces) cuts[p] = tokens_before(keys, n, piece_begin(rows + n, pieces, p));
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

struct PieceInfo { int64_t row; int32_t opened, closed; };     // first row of the piece; begun in an earlier piece; ends in this one

struct EmbedBwdParams {
    const uint32_t* keys; const uint32_t* perm; int64_t tokens, rows, cols;
    const void* dout; int64_t ld; void* out; int64_t ld_out; float scale;
    int32_t accumulate;
    int64_t pieces;
    const int64_t* cuts;                        // first token of each piece, [pieces + 1] (not where it accumulates)
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
    const int64_t piece = blockIdx.x, items = (P.accumulate ? 0 : P.rows) + P.tokens;
    const int64_t d0 = piece_begin(items, P.pieces, piece), d1 = piece_begin(items, P.pieces, piece + 1);
    const int64_t j0 = P.accumulate ? d0 : P.cuts[piece], j1 = P.accumulate ? d1 : P.cuts[piece + 1];
    const int64_t before = j0 > 0 ? (int64_t)P.keys[j0 - 1] : -1;   // row of the token before the piece
    int64_t r0, r1;                                            // rows that end in this piece: [r0, r1)
    if (P.accumulate) {
        r0 = j0 < j1 ? (int64_t)P.keys[j0] : P.rows;
        const int64_t last = j0 < j1 ? (int64_t)P.keys[j1 - 1] : -1;
        r1 = j1 < P.tokens && (int64_t)P.keys[j1] == last ? last : last + 1;
    } else {
        r0 = d0 - j0; r1 = d1 - j1;
    }
    r1 = r1 < P.rows ? r1 : P.rows;
    const bool opened = j0 < j1 || !P.accumulate ? before == r0 && r0 < P.rows : false;
    if (tid == 0 && blockIdx.y == 0) P.info[piece] = {r0, opened, r0 < r1};
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + tid) * N;
    const bool mine = c < P.cols;                              // N == 8: whole vectors
    const T* x = reinterpret_cast<const T*>(P.dout);
    O* out = reinterpret_cast<O*>(P.out);
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.0f;
    int64_t row = r0;                                          // the row being added up
    bool any = false;                                          // it has tokens in this piece
    auto close = [&]() {                                       // the row ends here
        if (mine) {
            if (row == r0 && opened) {
                store_cols<float, N>(P.head + piece * P.ld_part, c, acc);
            } else if (!P.accumulate || any) {
                float v[N];
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = acc[e] * P.scale;
                if (P.accumulate) {
                    float o[N];
                    load_cols<O, N>(out + row * P.ld_out, c, o);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] += o[e];
                }
                store_cols<O, N>(out + row * P.ld_out, c, v);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.0f;
        any = false;
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
                if (t + b < here && mine && skey[t + b] < P.rows) raw[b].load(x + (int64_t)sperm[t + b] * P.ld + c);
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (t + b >= here) break;
                const int64_t key = (int64_t)skey[t + b];
                if (key >= P.rows) break;                      // what has no gradient sorts last
                if (key != row) {
                    if (P.accumulate) { close(); row = key; }
                    else
                        for (; row < key; ++row) close();
                }
                float v[N];
                raw[b].values(v);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += v[e];
                any = true;
            }
        }
    }
    if (P.accumulate) {
        if (row < r1) { close(); row = P.rows; }
    } else {
        for (; row < r1; ++row) close();
    }
    if (any && mine) store_cols<float, N>(P.carry + piece * P.ld_part, c, acc);      // the row goes on in the next piece
}

// Rows that span pieces: the pieces' partial rows in order, by the CTA of the piece in which the row ends.
template <typename O, int N>
__global__ void __launch_bounds__(ROWS_THREADS) embedding_join_kernel(const EmbedBwdParams P) {
    pdl_enter();
    const int64_t piece = blockIdx.x;
    const PieceInfo me = P.info[piece];
    if (!me.opened || !me.closed) return;
    // Where the row begins: the last piece before this one that did not find it open.  Those between hold nothing else.  A warp looks
    // at 32 pieces at a time.
    int64_t first = piece - 1;
    for (;; first -= 32) {
        const int64_t p = first - (threadIdx.x & 31);
        const bool begins = p <= 0 || !(P.info[p].row == me.row && P.info[p].opened);
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, begins);
        if (who) { first -= __ffs(who) - 1; break; }
    }
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * N;
    if (c >= P.cols) return;
    float acc[N], v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.0f;
#pragma unroll 8
    for (int64_t p = first; p < piece; ++p) {
        load_cols<float, N>(P.carry + p * P.ld_part, c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += v[e];
    }
    load_cols<float, N>(P.head + piece * P.ld_part, c, v);
    O* o = reinterpret_cast<O*>(P.out) + me.row * P.ld_out;
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = (acc[e] + v[e]) * P.scale;
    if (P.accumulate) {
        load_cols<O, N>(o, c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += v[e];
    }
    store_cols<O, N>(o, c, acc);
}

// ------------------------------------------------------------------------------------------------
// workspace and launch
// ------------------------------------------------------------------------------------------------
// Pieces: enough for every SM to hold its share of CTAs, at least eight items each.  The bound does not ask the device, since the
// workspace's size is the same for every one.
constexpr int64_t MAX_PIECES = 1184;
static int64_t piece_count(int64_t items) {
    const int64_t n = (items + 7) / 8;
    return n < 1 ? 1 : n < MAX_PIECES ? n : MAX_PIECES;
}
static int64_t part_pitch(int64_t cols) { return (cols + 63) / 64 * 64; }
struct EmbedScratch { uint32_t* key[2]; uint32_t* place[2]; uint32_t* hist; int64_t* cuts; PieceInfo* info; float* carry; float* head; size_t bytes; };
static EmbedScratch embed_scratch(void* ws, int64_t tokens, int64_t rows, int64_t cols) {
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
    const int64_t pieces = piece_count(rows + tokens);
    s.cuts = (int64_t*)take((size_t)(pieces + 1) * 8);
    s.info = (PieceInfo*)take((size_t)pieces * sizeof(PieceInfo));
    s.carry = (float*)take((size_t)pieces * part_pitch(cols) * 4);
    s.head = (float*)take((size_t)pieces * part_pitch(cols) * 4);
    s.bytes = at;
    return s;
}
size_t embedding_bytes(int64_t tokens, int64_t rows, int64_t cols) { return embed_scratch(nullptr, tokens, rows, cols).bytes; }

template <typename T, typename O>
static cudaError_t launch_rows(const EmbedBwdParams& P, bool vec, cudaStream_t st) {
    const int64_t n = vec ? P.cols / 8 : P.cols;
    const int threads = n >= ROWS_THREADS ? ROWS_THREADS : (int)((n + 31) / 32 * 32);
    const dim3 grid((unsigned)P.pieces, (unsigned)((n + threads - 1) / threads)), block(threads);
    count_launch();
    cudaError_t e = vec ? launch_pdl(embedding_rows_kernel<T, O, 8>, grid, block, 0, st, P) : launch_pdl(embedding_rows_kernel<T, O, 1>, grid, block, 0, st, P);
    if (e != cudaSuccess || P.pieces == 1) return e;
    count_launch();
    return vec ? launch_pdl(embedding_join_kernel<O, 8>, grid, block, 0, st, P) : launch_pdl(embedding_join_kernel<O, 1>, grid, block, 0, st, P);
}

cudaError_t launch_embedding_bwd(const EmbedBwdArgs& a, cudaStream_t st) {
    const EmbedScratch s = embed_scratch(a.ws, a.tokens, a.rows, a.cols);
    const SortPlan plan = sort_plan(a.rows);
    const int64_t pieces = piece_count((a.accumulate ? 0 : a.rows) + a.tokens);
    const int wide = a.id_t == SRQ_I64;
    int last = 0;                                              // buffers that hold the sorted tokens
    if (a.tokens > 0 && a.tokens <= SORT_ONE) {
        cudaError_t e = cudaFuncSetAttribute(sort_one_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortOneShared));
        if (e != cudaSuccess) return e;
        count_launch();
        e = launch_pdl(sort_one_kernel, dim3(1), dim3(SORT_ONE_THREADS), sizeof(SortOneShared), st, a.ids, wide, (int)a.tokens, a.rows, plan.total, s.key[0], s.place[0],
                       a.accumulate ? (int64_t*)nullptr : s.cuts, pieces, a.status);
        if (e != cudaSuccess) return e;
    } else if (a.tokens > 0) {
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
    if ((a.tokens == 0 || a.tokens > SORT_ONE) && !a.accumulate) {
        count_launch();
        const cudaError_t e = launch_pdl(cut_kernel, dim3((unsigned)(pieces / 256 + 1)), dim3(256), 0, st, (const uint32_t*)s.key[last], a.tokens, a.rows, s.cuts, pieces);
        if (e != cudaSuccess) return e;
    }
    EmbedBwdParams P;
    P.keys = s.key[last]; P.perm = s.place[last]; P.tokens = a.tokens; P.rows = a.rows; P.cols = a.cols;
    P.dout = a.dout; P.ld = a.ld; P.out = a.out; P.ld_out = a.ld_out; P.scale = a.scale; P.accumulate = a.accumulate;
    P.pieces = pieces; P.cuts = s.cuts;
    P.info = s.info; P.carry = s.carry; P.head = s.head; P.ld_part = part_pitch(a.cols);
    const bool vec = whole_vectors(a.dout, a.ld, a.cols, a.dt) && whole_vectors(a.out, a.ld_out, a.cols, a.out_dt);
    typedef __nv_bfloat16 H;
    if (a.dt == SRQ_F32) return a.out_dt == SRQ_F32 ? launch_rows<float, float>(P, vec, st) : launch_rows<float, H>(P, vec, st);
    return a.out_dt == SRQ_F32 ? launch_rows<H, float>(P, vec, st) : launch_rows<H, H>(P, vec, st);
}

}  // namespace srq
