// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Forward: a copy of rows; bound by HBM (rows that come up often are read from L2).
//
// Gradient.  The tokens are sorted by id (stable, radix), so that the tokens of one row of the table are neighbours, in the order
// in which they came.  The rows of the table and the sorted tokens are then merged into one list (a row's tokens, then the row's end)
// and cut into equal pieces, one per CTA: the merge path of sparse products (Merrill and Garland, SC'16), which gives
// every CTA the same number of rows to write and tokens to add, however uneven the ids are.  Item j of the sorted tokens stands
// at place j + id_j of the list, so that a cut is found by one search.  A CTA writes the rows that end in its piece, zero rows
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

// N elements of a row as they lie in memory (eight: 16-byte aligned).
template <typename T, int N> struct alignas(N == 8 ? 16 : sizeof(T)) Raw { T e[N]; };
template <typename T, int N>
__device__ __forceinline__ void values(const Raw<T, N>& r, float v[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)r.e[e];
}

// VEC: eight elements of a row at a time, else one.
template <typename I, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(const EmbedFwdParams P) {
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
        raw[u] = {};
        if (valid && c0 + u * step < P.cols) raw[u] = *reinterpret_cast<const Raw<I, N>*>(src + c0 + u * step);
    }
#pragma unroll
    for (int u = 0; u < EMBED_U; ++u) {
        const int64_t c = c0 + u * step;
        if (c >= P.cols) break;
        float v[N];
        values<I, N>(raw[u], v);
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
// Digits of at most 9 bits, lowest first.  Keys are ids; everything without a gradient has the key `rows`, which sorts last.
constexpr int SORT_BINS = 512, SORT_ONE = 16384, SORT_ONE_THREADS = 1024, SORT_TILE = 4096, SORT_THREADS = 512, SORT_MAX_BLOCKS = 128;

struct SortPlan { int passes, bits; };
static SortPlan sort_plan(int64_t rows) {
    int bits = 1;
    while (bits < 31 && ((int64_t)1 << bits) <= rows) ++bits;  // keys 0 .. rows
    SortPlan p;
    p.passes = (bits + 8) / 9;
    p.bits = (bits + p.passes - 1) / p.passes;
    return p;
}

__device__ __forceinline__ uint32_t key_of(const void* ids, int wide, int64_t i, int64_t rows, uint32_t* status) {
    const int64_t id = whole_at(ids, wide, i);
    if (id >= rows) note(status, SRQ_ERR_INVALID_ARG);
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

// Ranks a warp's keys, 32 at a time in their order: place among the warp's keys of the same digit so far.  counts: the warp's own.
// Who has the same digit is found by a ballot per bit (the instruction that matches whole words is an order slower: 16384 tokens 41 us).
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
    uint32_t base = 0;
    for (int w = 0; w < warp; ++w) base += warp_sums[w];
    __syncthreads();
    return base + s - x;
}

// All passes in one CTA, for up to SORT_ONE tokens.  Shared memory: keys, places (16 bits), a counter per warp and bin.
struct SortOneShared {
    uint32_t key[SORT_ONE];
    uint16_t place[SORT_ONE];
    uint16_t count[SORT_ONE_THREADS / 32][SORT_BINS];
    uint32_t base[SORT_BINS];
    uint32_t sums[32];
};
__global__ void __launch_bounds__(SORT_ONE_THREADS) sort_one_kernel(const void* ids, int wide, int n, int64_t rows, SortPlan plan, uint32_t* keys, uint32_t* perm,
                                                                    uint32_t* status) {
    pdl_enter();
    extern __shared__ char raw[];
    SortOneShared& S = *reinterpret_cast<SortOneShared*>(raw);
    constexpr int MOST = SORT_ONE / SORT_ONE_THREADS, WARPS = SORT_ONE_THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int turns = (n + SORT_ONE_THREADS - 1) / SORT_ONE_THREADS, first = warp * turns * 32 + lane;
    for (int i = tid; i < n; i += SORT_ONE_THREADS) { S.key[i] = key_of(ids, wide, i, rows, status); S.place[i] = (uint16_t)i; }
    for (int pass = 0; pass < plan.passes; ++pass) {
        const int shift = pass * plan.bits, bins = 1 << plan.bits;
        const uint32_t mask = (uint32_t)bins - 1u;
        uint32_t key[MOST], rank[MOST];                        // rank: place in the upper half
        for (int i = tid; i < WARPS * SORT_BINS / 2; i += SORT_ONE_THREADS) reinterpret_cast<uint32_t*>(&S.count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MOST; ++t) {
            if (t >= turns) break;
            const int i = first + t * 32;
            const bool active = i < n;
            key[t] = active ? S.key[i] : 0u;
            rank[t] = active ? (uint32_t)S.place[i] << 16 : 0u;
            rank[t] |= rank_in_warp((key[t] >> shift) & mask, plan.bits, active, S.count[warp], lane);
        }
        __syncthreads();
        uint32_t total = 0;
        if (tid < bins) {
            for (int w = 0; w < WARPS; ++w) { const uint32_t c = S.count[w][tid]; S.count[w][tid] = (uint16_t)total; total += c; }
        }
        const uint32_t base = exclusive_scan<SORT_ONE_THREADS>(total, S.sums);
        if (tid < bins) S.base[tid] = base;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MOST; ++t) {
            if (t >= turns) break;
            if (first + t * 32 < n) {
                const uint32_t d = (key[t] >> shift) & mask, to = S.base[d] + S.count[warp][d] + (rank[t] & 0xFFFFu);
                S.key[to] = key[t];
                S.place[to] = (uint16_t)(rank[t] >> 16);
            }
        }
        __syncthreads();
    }
    for (int i = tid; i < n; i += SORT_ONE_THREADS) { keys[i] = S.key[i]; perm[i] = S.place[i]; }
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
    for (int64_t i = first + tid; i < end; i += SORT_THREADS) {
        const uint32_t k = P.ids ? key_of(P.ids, P.wide, i, P.rows, P.status) : P.key_in[i];
        atomicAdd(&count[(k >> P.shift) & mask], 1u);
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
        for (int i = tid; i < WARPS * SORT_BINS / 2; i += SORT_THREADS) reinterpret_cast<uint32_t*>(&count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t i = tile + (warp * TURNS + t) * 32 + lane;
            const bool active = i < end;
            key[t] = !active ? 0u : P.ids ? key_of(P.ids, P.wide, i, P.rows, nullptr) : P.key_in[i];
            rank[t] = rank_in_warp((key[t] >> P.shift) & mask, P.bits, active, count[warp], lane);
        }
        __syncthreads();
        uint32_t here = 0;
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
constexpr int ROWS_THREADS = 256, ROWS_BATCH = 4;

struct PieceInfo { int64_t row; int32_t opened, closed; };     // first row of the piece; begun in an earlier piece; ends in this one

struct EmbedBwdParams {
    const uint32_t* keys; const uint32_t* perm; int64_t tokens, rows, cols;
    const void* dout; int64_t ld; void* out; int64_t ld_out; float scale;
    int32_t accumulate;
    int64_t pieces;
    PieceInfo* info; float* carry; float* head; int64_t ld_part;   // partial rows [pieces, ld_part]: at the end, at the beginning
};

// Tokens before place d of the merged list: the first j with j + key_j >= d.  One warp; 32 probes a step.
__device__ __forceinline__ int64_t tokens_before(const uint32_t* keys, int64_t n, int64_t d, int lane) {
    int64_t lo = 0, hi = n;                                    // answer in [lo, hi]
    while (hi > lo) {
        const int64_t step = (hi - lo + 31) / 32, j = lo + lane * step;
        const bool less = j < hi && j + (int64_t)keys[j] < d;
        const int c = __popc(__ballot_sync(0xFFFFFFFFu, less));    // the probes that are less come first
        if (c == 0) return lo;
        const int64_t nlo = lo + (c - 1) * step + 1;
        hi = lo + c * step < hi ? lo + c * step : hi;
        lo = nlo;
    }
    return lo;
}

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
__global__ void __launch_bounds__(ROWS_THREADS) embedding_rows_kernel(const EmbedBwdParams P) {
    pdl_enter();
    __shared__ int64_t cut[2];
    __shared__ uint32_t skey[ROWS_THREADS], sperm[ROWS_THREADS];
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t piece = blockIdx.x, items = (P.accumulate ? 0 : P.rows) + P.tokens;
    const int64_t d0 = items / P.pieces * piece + (items % P.pieces) * piece / P.pieces;
    const int64_t d1 = items / P.pieces * (piece + 1) + (items % P.pieces) * (piece + 1) / P.pieces;
    if (P.accumulate) {
        if (tid < 2) cut[tid] = tid ? d1 : d0;
    } else if (tid < 32) {
        const int64_t a = tokens_before(P.keys, P.tokens, d0, lane), b = tokens_before(P.keys, P.tokens, d1, lane);
        if (lane == 0) { cut[0] = a; cut[1] = b; }
    }
    __syncthreads();
    const int64_t j0 = cut[0], j1 = cut[1];
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
        for (int t = 0; t < here; t += ROWS_BATCH) {
            float v[ROWS_BATCH][N];
#pragma unroll
            for (int b = 0; b < ROWS_BATCH; ++b) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[b][e] = 0.0f;
                if (t + b < here && mine && skey[t + b] < P.rows) load_cols<T, N>(x + (int64_t)sperm[t + b] * P.ld, c, v[b]);
            }
#pragma unroll
            for (int b = 0; b < ROWS_BATCH; ++b) {
                if (t + b >= here) break;
                const int64_t key = (int64_t)skey[t + b];
                if (key >= P.rows) break;                      // what has no gradient sorts last
                if (P.accumulate) {
                    if (key != row) { close(); row = key; }
                } else {
                    for (; row < key; ++row) close();
                }
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += v[b][e];
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
struct EmbedScratch { uint32_t* key[2]; uint32_t* place[2]; uint32_t* hist; PieceInfo* info; float* carry; float* head; size_t bytes; };
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
    const int wide = a.id_t == SRQ_I64;
    int last = 0;                                              // buffers that hold the sorted tokens
    if (a.tokens > 0 && a.tokens <= SORT_ONE) {
        cudaError_t e = cudaFuncSetAttribute(sort_one_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortOneShared));
        if (e != cudaSuccess) return e;
        count_launch();
        e = launch_pdl(sort_one_kernel, dim3(1), dim3(SORT_ONE_THREADS), sizeof(SortOneShared), st, a.ids, wide, (int)a.tokens, a.rows, plan, s.key[0], s.place[0], a.status);
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
    EmbedBwdParams P;
    P.keys = s.key[last]; P.perm = s.place[last]; P.tokens = a.tokens; P.rows = a.rows; P.cols = a.cols;
    P.dout = a.dout; P.ld = a.ld; P.out = a.out; P.ld_out = a.ld_out; P.scale = a.scale; P.accumulate = a.accumulate;
    P.pieces = piece_count((a.accumulate ? 0 : a.rows) + a.tokens);
    P.info = s.info; P.carry = s.carry; P.head = s.head; P.ld_part = part_pitch(a.cols);
    const bool vec = whole_vectors(a.dout, a.ld, a.cols, a.dt) && whole_vectors(a.out, a.ld_out, a.cols, a.out_dt);
    typedef __nv_bfloat16 H;
    if (a.dt == SRQ_F32) return a.out_dt == SRQ_F32 ? launch_rows<float, float>(P, vec, st) : launch_rows<float, H>(P, vec, st);
    return a.out_dt == SRQ_F32 ? launch_rows<H, float>(P, vec, st) : launch_rows<H, H>(P, vec, st);
}

}  // namespace srq
