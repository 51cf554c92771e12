// Block-scaled E4M3 quantizer (1 x 128 blocks or 128 x 128 tiles, row-major and / or transposed) and the
// backward pass of the gated feed-forward block, which is the same kernel over values it computes itself.
//
// 128 x 128 tiles, 512 threads per CTA, persistent CTAs.  Thread (g, l), g = 0..31, l = 0..15, holds rows
// 4 g .. 4 g + 3 of columns 8 l .. 8 l + 7 in registers, so that
//   - a row's 128 values sit in 16 neighbouring lanes: the absmax of four rows is a butterfly of five shuffles that leaves
//     row l % 4's in lane l;
//   - a column's 128 values sit in the warps' lanes l and l + 16: its absmax is half a shuffle and half a shared atomic;
//   - the transposed codes of a thread are 8 words of 4 bytes, which meet in a swizzled shared tile.
// (Two rows per thread and 1024 threads were measured too: twice the warps, but 69 instead of 57 instructions per value,
// and no faster.)
// A tile is read once whatever is written: both layouts and both kinds of step size come from the registers.
// While a tile is worked on, the next one is on its way into shared memory (cp.async, 16 bytes at a time: smaller
// pieces were measured to cost a shared-memory wavefront per lane); tiles that reach over the matrix's edge, and sources
// whose alignment does not allow it, are read directly with bounds checks.
// The kernels are bound by instruction issue as much as by HBM, hence the two-at-a-time binary32 instructions.
#include <mutex>
#include <type_traits>

#include "blocks.cuh"

namespace srq {

constexpr int TQ_THREADS = 512;
constexpr int R = 4;                     // rows per thread

// NOUT matrices are quantized from one tile (1, or the three of the gated block's backward pass).
template <int NOUT>
struct TileShared {
    uint32_t col_max[2][NOUT][QBLK];     // [tile parity][matrix][column % 4][column / 4 % 2][column / 8]: an atomic per lane and bank
    alignas(8) float col_inv[NOUT][QBLK];          // [column % 8 / 2][column / 8][column % 2]: read two by two
    uint32_t tile_max[2];
    alignas(16) uint32_t words[NOUT][QBLK * 32];   // transposed codes: column c's rows 4 g .. 4 g + 3 at [c][g ^ 2 (c / 8)]
};

struct TilePos {
    int64_t r0, c0;                      // tile origin
    bool full;                           // inside the matrix and read ahead through shared memory
};

__device__ __forceinline__ TilePos tile_at(uint32_t tile, uint32_t tiles_c, int64_t rows, int64_t cols, int vec) {
    TilePos p;
    const uint32_t tr = tile / tiles_c;
    p.r0 = (int64_t)tr * QBLK;
    p.c0 = (int64_t)(tile - tr * tiles_c) * QBLK;
    p.full = vec && p.r0 + QBLK <= rows && p.c0 + QBLK <= cols;
    return p;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ uint32_t shared_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Read-ahead shared memory: a matrix's tile in one buffer (bfloat16: each thread its own values; binary32: a row's 16-byte
// chunks lane by lane, since a thread's own eight values are two chunks and every sector would be asked for twice,
// so the next tile is asked for only when every thread has read its share); a block-coded matrix's tile row by
// row, and its rows' step sizes (two buffers each, in turn).
template <typename T> __host__ __device__ constexpr int matrix_slot() { return QBLK * QBLK * (int)sizeof(T); }
constexpr int CODED_TILE = QBLK * QBLK;
__host__ __device__ constexpr int coded_slot() { return 2 * (CODED_TILE + QBLK * 4); }

// Thread's share of a matrix / a block-coded matrix: into shared memory ahead of time, and from there (ahead) or
// from global memory (with bounds checks) into registers.
template <typename T>
__device__ __forceinline__ void fetch_matrix(uint8_t* slot, const T* x, int64_t ld, const TilePos& p) {
    if constexpr (sizeof(T) == 4) {
        const int k = threadIdx.x & 31, row = threadIdx.x >> 5;            // chunk k of rows row, row + 64 / R, ...
        const T* src = x + (p.r0 + row) * ld + p.c0 + 4 * k;
        // neighbouring chunks change places in every other group of eight: a thread's two reads hit all banks
        const uint32_t dst = shared_addr(slot) + row * 512 + ((k ^ ((k >> 3) & 1)) << 4);
#pragma unroll
        for (int i = 0; i < 2 * R; ++i, src += (64 / R) * ld) cp_async16(dst + i * (64 / R) * 512, src);
    } else {
        const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
        const T* src = x + (p.r0 + R * g) * ld + p.c0 + 8 * l;
        const uint32_t dst = shared_addr(slot) + threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < R; ++i, src += ld) cp_async16(dst + i * TQ_THREADS * 16, src);
    }
}
template <typename T>
__device__ __forceinline__ void read_matrix(const uint8_t* slot, const T* x, int64_t ld, int64_t rows, int64_t cols, int vec, const TilePos& p, float (&v)[R][8]) {
    const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (p.full) {
            const uint4* s = reinterpret_cast<const uint4*>(slot) + threadIdx.x;
            if constexpr (sizeof(T) == 4) {
                const uint4* row = reinterpret_cast<const uint4*>(slot) + (R * g + i) * 32;
                const uint4 a = row[(2 * l) ^ ((l >> 2) & 1)], b = row[(2 * l + 1) ^ ((l >> 2) & 1)];
                v[i][0] = __uint_as_float(a.x); v[i][1] = __uint_as_float(a.y); v[i][2] = __uint_as_float(a.z); v[i][3] = __uint_as_float(a.w);
                v[i][4] = __uint_as_float(b.x); v[i][5] = __uint_as_float(b.y); v[i][6] = __uint_as_float(b.z); v[i][7] = __uint_as_float(b.w);
            } else {
                const uint4 a = s[i * TQ_THREADS];
                v[i][0] = bf16_lo(a.x); v[i][1] = bf16_hi(a.x); v[i][2] = bf16_lo(a.y); v[i][3] = bf16_hi(a.y);
                v[i][4] = bf16_lo(a.z); v[i][5] = bf16_hi(a.z); v[i][6] = bf16_lo(a.w); v[i][7] = bf16_hi(a.w);
            }
        } else {
            const int64_t r = p.r0 + R * g + i;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
            if (r < rows) load8(x + r * ld, p.c0 + 8 * l, cols, vec, v[i]);
        }
    }
}
__device__ __forceinline__ void fetch_coded(uint8_t* slot, const Blocks& b, const TilePos& p) {
    const int row = threadIdx.x >> 3, q = threadIdx.x & 7;             // eight threads to a row's 128 codes
    const uint8_t* src = b.codes + (p.r0 + row) * b.ld + p.c0 + 16 * q;
    const uint32_t dst = shared_addr(slot) + row * QBLK + 16 * q;
#pragma unroll
    for (int i = 0; i < R / 2; ++i) cp_async16(dst + i * 64 * QBLK, src + i * 64 * b.ld);
}
// The step size of row `row` of a tile, on its way to coded_scales() of its buffer.
__device__ __forceinline__ float fetch_scale(const Blocks& b, const TilePos& p, int row) {
    return b.scale[(b.tile_rows > 1 ? p.r0 / QBLK : p.r0 + row) * b.ld_scale + p.c0 / QBLK];
}
__device__ __forceinline__ uint8_t* coded_codes(uint8_t* slot, int par) { return slot + par * CODED_TILE; }
__device__ __forceinline__ float* coded_scales(uint8_t* slot, int par) { return reinterpret_cast<float*>(slot + 2 * CODED_TILE) + par * QBLK; }

__device__ __forceinline__ void read_coded(uint8_t* slot, int par, const Blocks& b, int64_t rows, int64_t cols, const TilePos& p, float (&v)[R][8]) {
    const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        uint2 w = make_uint2(0u, 0u);
        float s = 0.0f;
        if (p.full) {
            w = *reinterpret_cast<const uint2*>(coded_codes(slot, par) + (R * g + i) * QBLK + 8 * l);
            s = coded_scales(slot, par)[R * g + i];
        } else {
            const int64_t r = p.r0 + R * g + i, c = p.c0 + 8 * l;
            if (r < rows && c < cols) {
                const uint8_t* row = b.codes + r * b.ld;
                if (c + 8 <= cols) w = *reinterpret_cast<const uint2*>(row + c);
                else
                    for (int e = 0; e < 8; ++e)
                        if (c + e < cols) (e < 4 ? w.x : w.y) |= (uint32_t)row[c + e] << (8 * (e & 3));
                s = b.scale[(b.tile_rows > 1 ? r / QBLK : r) * b.ld_scale + c / QBLK];
            }
        }
        e4m3x4_to_f32(w.x, v[i]);
        e4m3x4_to_f32(w.y, v[i] + 4);
        const float2 s2 = make_float2(s, s);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float2 y = __fmul2_rn(make_float2(v[i][e], v[i][e + 1]), s2);
            v[i][e] = y.x; v[i][e + 1] = y.y;
        }
    }
}

template <int NOUT>
struct TileOut {
    Blocks rm[NOUT], tr[NOUT];           // codes == nullptr: not wanted
    int64_t rows, cols;
    uint64_t index_offset;
    PhiloxKeys keys[NOUT];
    const int64_t* step;                 // of BlockRounding
    uint32_t* status;
};

// Quantizes the NOUT matrices whose tile is held as v (zeros outside the matrix).  All threads of the CTA call it
// together, after a barrier that follows the previous call; `next` asks for the next tile; later: step_word().
template <int NOUT, bool SR, bool FULL, typename Next>
__device__ __forceinline__ void emit_tile(const float (&v)[NOUT][R][8], const TileOut<NOUT>& O, const TilePos& p, int par,
                                          TileShared<NOUT>* S, uint32_t later, Next&& next) {
    const int tid = threadIdx.x, lane = tid & 31, l = tid & 15, g = tid >> 4;
    const int64_t r_first = p.r0 + R * g, c_first = p.c0 + 8 * l;
    bool any_tr = false, tiles = false;
#pragma unroll
    for (int n = 0; n < NOUT; ++n) {
        any_tr |= O.tr[n].codes != nullptr;
        tiles |= (O.rm[n].codes && O.rm[n].tile_rows > 1) || (O.tr[n].codes && O.tr[n].tile_rows > 1);
    }
    const bool meet = any_tr || tiles;
    next();
    // ---- maxima
    uint32_t row_max[NOUT] = {};         // of row l % R
#pragma unroll
    for (int n = 0; n < NOUT; ++n) {
        const bool tile_n = NOUT == 1 && tiles;            // 128 x 128 tiles: the quantizer only
        if (O.rm[n].codes || tile_n) {
            uint32_t m[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float (&x)[8] = v[n][i];
                m[i] = abs_word(absmax3(absmax3(x[0], x[1], x[2]), absmax3(x[3], x[4], x[5]), absmax3(x[6], x[7], 0.0f)));
            }
            // halve the rows, then the lanes: lane l keeps the rows whose low bits agree with its own
#pragma unroll
            for (int w = 1; w < R; w <<= 1) {
                const bool odd = (l & w) != 0;
#pragma unroll
                for (int i = 0; i < R / (2 * w); ++i) {
                    const uint32_t keep = odd ? m[2 * i + 1] : m[2 * i], give = odd ? m[2 * i] : m[2 * i + 1];
                    m[i] = max(keep, __shfl_xor_sync(0xFFFFFFFFu, give, w));
                }
            }
#pragma unroll
            for (int w = R; w < 16; w <<= 1) m[0] = max(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], w));
            row_max[n] = m[0];
        }
        if (tile_n) {
            const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, row_max[n]);
            if (lane == 0) atomicMax(&S->tile_max[par], m);
        }
        if (O.tr[n].codes && O.tr[n].tile_rows == 1) {
            uint32_t m[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                m[j] = abs_word(absmax3(absmax3(v[n][0][j], v[n][1][j], v[n][2][j]), v[n][3][j], 0.0f));
            const int b = lane >> 4;                       // lanes 0 - 15 finish columns 0 - 3 of the eight, the others 4 - 7
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t keep = b ? m[j + 4] : m[j], give = b ? m[j] : m[j + 4];
                atomicMax(&S->col_max[par][n][j * 32 + lane], max(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 16)));
            }
        }
    }
    if (meet) {
        __syncthreads();
        // ---- columns' step sizes, and the other parity's maxima back to zero for the next tile
        for (int t = tid; t < NOUT * QBLK; t += TQ_THREADS) {
            const int n = t / QBLK, k = t & (QBLK - 1);
            const Blocks& o = O.tr[n];
            S->col_max[par ^ 1][n][k] = 0u;
            if (t == 0) S->tile_max[par ^ 1] = 0u;
            if (!o.codes) continue;
            const int kl = k & 15, kj = (k >> 5) + ((k >> 4) & 1) * 4;      // column 8 kl + kj of the tile
            const int64_t c = p.c0 + 8 * kl + kj;
            const bool tile = o.tile_rows > 1;
            const uint32_t m = tile ? S->tile_max[par] : S->col_max[par][n][k];
            S->col_inv[n][(kj >> 1) * 32 + kl * 2 + (kj & 1)] = block_inv(m);
            if (block_nonfinite(m)) note(O.status, SRQ_ERR_NONFINITE);
            if (!tile && (FULL || c < O.cols)) o.scale[c * o.ld_scale + p.r0 / QBLK] = block_size(m);
            if (tile && k == 0) o.scale[(p.c0 / QBLK) * o.ld_scale + p.r0 / QBLK] = block_size(m);
        }
    }
    // ---- row-major codes
#pragma unroll
    for (int n = 0; n < NOUT; ++n) {
        const Blocks& o = O.rm[n];
        if (!o.codes) continue;
        const bool tile = NOUT == 1 && o.tile_rows > 1;
        // a division per thread: lane l has its row l % R's absmax
        const uint32_t m = tile ? S->tile_max[par] : row_max[n];
        const float inv = block_inv(m);
        if (block_nonfinite(m)) note(O.status, SRQ_ERR_NONFINITE);
        const int64_t r_mine = r_first + (l & (R - 1));
        if (!tile && l < R && (FULL || r_mine < O.rows)) o.scale[r_mine * o.ld_scale + p.c0 / QBLK] = block_size(m);
        if (tile && tid == 0) o.scale[(p.r0 / QBLK) * o.ld_scale + p.c0 / QBLK] = block_size(m);
        uint8_t* dst = o.codes + r_first * o.ld + c_first;
#pragma unroll
        for (int i = 0; i < R; ++i, dst += o.ld) {
            const float f = __shfl_sync(0xFFFFFFFFu, inv, (lane & 16) + i);
            const float (&x)[8] = v[n][i];
            uint32_t rnd[8] = {};
            if constexpr (SR) thresholds8(O.index_offset + (uint64_t)(r_first + i) * (uint64_t)O.cols + (uint64_t)c_first, O.keys[n], later, rnd);
            const uint32_t w0 = encode4<SR>(x[0], x[1], x[2], x[3], f, f, f, f, rnd[0], rnd[1], rnd[2], rnd[3]);
            const uint32_t w1 = encode4<SR>(x[4], x[5], x[6], x[7], f, f, f, f, rnd[4], rnd[5], rnd[6], rnd[7]);
            if (FULL) *reinterpret_cast<uint2*>(dst) = make_uint2(w0, w1);
            else if (r_first + i < O.rows && c_first < O.cols) store_codes8(dst - c_first, c_first, O.cols, w0, w1);
        }
    }
    if (!any_tr) return;
    // ---- transposed codes, through shared memory
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NOUT; ++n) {
        if (!O.tr[n].codes) continue;
        uint32_t* words = S->words[n] + (8 * l) * 32 + (g ^ (2 * l));
        if constexpr (SR) {
            uint32_t w[8] = {};
#pragma unroll
            for (int i = 0; i < R; ++i) {                  // a row's thresholds at a time
                uint32_t rnd[8];
                thresholds8(O.index_offset + (uint64_t)(r_first + i) * (uint64_t)O.cols + (uint64_t)c_first, O.keys[n], later, rnd);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    w[j] |= (quantize_e4m3<MODE_SR | MODE_E4M3>(v[n][i][j], S->col_inv[n][(j >> 1) * 32 + 2 * l + (j & 1)], rnd[j], 0) & 0xFFu) << (8 * i);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) words[j * 32] = w[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 f = *reinterpret_cast<const float2*>(&S->col_inv[n][(j >> 1) * 32 + 2 * l]);
                float2 t[R];
#pragma unroll
                for (int i = 0; i < R; ++i) t[i] = __fmul2_rn(make_float2(v[n][i][j], v[n][i][j + 1]), f);
                words[j * 32] = e4m3x4(t[0].x, t[1].x, t[2].x, t[3].x);
                words[(j + 1) * 32] = e4m3x4(t[0].y, t[1].y, t[2].y, t[3].y);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NOUT; ++n) {
        const Blocks& o = O.tr[n];
        if (!o.codes) continue;
        if (FULL) {
            // sixteen codes per store: chunk q of column c; its four words sit in chunk q ^ (l / 2), halves swapped for odd l
            // (l = c / 8)
            const int q = tid & 7;
#pragma unroll
            for (int h = 0; h < R / 2; ++h) {
                const int cc = (tid >> 3) + 64 * h, lc = cc >> 3;
                const uint4 w = *reinterpret_cast<const uint4*>(&S->words[n][cc * 32 + ((q ^ (lc >> 1)) << 2)]);
                *reinterpret_cast<uint4*>(o.codes + (p.c0 + cc) * o.ld + p.r0 + 16 * q) = (lc & 1) ? make_uint4(w.z, w.w, w.x, w.y) : w;
            }
        } else {
            const int64_t r = p.r0 + 4 * lane;
#pragma unroll 1
            for (int k = 0; k < 2 * R; ++k) {
                const int cc = 2 * R * (tid >> 5) + k;
                const int64_t c = p.c0 + cc;
                if (c >= O.cols || r >= O.rows) continue;
                const uint32_t w = S->words[n][cc * 32 + (lane ^ (2 * (cc >> 3)))];
                uint8_t* dst = o.codes + c * o.ld + r;
                if (r + 4 <= O.rows) *reinterpret_cast<uint32_t*>(dst) = w;
                else
                    for (int e = 0; e < 4 && r + e < O.rows; ++e) dst[e] = (uint8_t)(w >> (8 * e));
            }
        }
    }
}

template <int NOUT>
__device__ __forceinline__ void clear_maxima(TileShared<NOUT>* S) {
    for (int t = threadIdx.x; t < 2 * NOUT * QBLK; t += blockDim.x) S->col_max[0][0][t] = 0u;
    if (threadIdx.x < 2) S->tile_max[threadIdx.x] = 0u;
}

struct QuantBlocksParams {
    BlockSource src;
    TileOut<1> out;
    uint32_t tiles, tiles_c;
    int32_t vec;                         // the source's alignment allows 16-byte (codes: 8-byte) accesses
};

// SRC: 0 binary32, 1 bfloat16, 2 block codes.
template <int SRC, bool SR>
__global__ void __launch_bounds__(TQ_THREADS, 2 - SR) quantize_blocks_kernel(const __grid_constant__ QuantBlocksParams P) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t ahead[];
    __shared__ TileShared<1> S;
    using T = std::conditional_t<SRC == 0, float, __nv_bfloat16>;
    const int64_t rows = P.out.rows, cols = P.out.cols;
    const uint32_t later = SR ? step_word(P.out.step) : 0u;
    int par = 0;
    auto fetch = [&](const TilePos& p, int to) {
        if (p.full) {
            if constexpr (SRC == 2) fetch_coded(coded_codes(ahead, to), P.src.coded, p);
            else fetch_matrix<T>(ahead, (const T*)P.src.x, P.src.ld, p);
        }
        cp_async_commit();
    };
    clear_maxima(&S);
    TilePos p = tile_at(blockIdx.x, P.tiles_c, rows, cols, P.vec);
    fetch(p, 0);
    if (SRC == 2 && threadIdx.x < QBLK && p.full) coded_scales(ahead, 0)[threadIdx.x] = fetch_scale(P.src.coded, p, threadIdx.x);
#pragma unroll 1
    for (uint32_t tile = blockIdx.x; tile < P.tiles; par ^= 1) {
        float v[1][4][8];
        cp_async_wait();
        __syncthreads();                 // everybody's pieces have landed, the last tile's shared words have been read
        if constexpr (SRC == 2) read_coded(ahead, par, P.src.coded, rows, cols, p, v[0]);
        else read_matrix<T>(ahead, (const T*)P.src.x, P.src.ld, rows, cols, P.vec, p, v[0]);
        const uint32_t next_tile = tile + gridDim.x;
        const TilePos np = tile_at(next_tile < P.tiles ? next_tile : tile, P.tiles_c, rows, cols, P.vec);
        float next_scale = 0.0f;
        auto next = [&] {
            if (SRC == 0) __syncthreads();
            if (next_tile >= P.tiles) return;
            fetch(np, par ^ 1);
            if (SRC == 2 && threadIdx.x < QBLK && np.full) next_scale = fetch_scale(P.src.coded, np, threadIdx.x);
        };
        if (p.full) emit_tile<1, SR, true>(v, P.out, p, par, &S, later, next);
        else emit_tile<1, SR, false>(v, P.out, p, par, &S, later, next);
        if (SRC == 2 && threadIdx.x < QBLK) coded_scales(ahead, par ^ 1)[threadIdx.x] = next_scale;
        tile = next_tile;
        p = np;
    }
}

struct GluBwdParams {
    const void* dh; int64_t ld_dh;
    Blocks gate, up;
    TileOut<3> out;                      // dg, du, h
    uint32_t tiles, tiles_c;
    int32_t vec;
};

// dg = dh u act'(g), du = dh act(g), h = act(g) u over a tile, all three formed with one evaluation of the activation.
template <typename T, bool GELU, bool SR>
__global__ void __launch_bounds__(TQ_THREADS, 1) glu_bwd_kernel(const __grid_constant__ GluBwdParams P) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t dyn[];
    TileShared<3>* S = reinterpret_cast<TileShared<3>*>(dyn);
    uint8_t* ahead_dh = dyn + (sizeof(TileShared<3>) + 15) / 16 * 16;
    uint8_t* ahead_g = ahead_dh + matrix_slot<T>();
    uint8_t* ahead_u = ahead_g + coded_slot();
    const int64_t rows = P.out.rows, cols = P.out.cols;
    const uint32_t later = SR ? step_word(P.out.step) : 0u;
    int par = 0;
    auto fetch = [&](const TilePos& p, int to) {
        if (p.full) {
            fetch_matrix<T>(ahead_dh, (const T*)P.dh, P.ld_dh, p);
            fetch_coded(coded_codes(ahead_g, to), P.gate, p);
            fetch_coded(coded_codes(ahead_u, to), P.up, p);
        }
        cp_async_commit();
    };
    // threads 0 .. 127 bring the rows' step sizes of the gate, the next 128 those of the up projection
    uint8_t* scale_slot = threadIdx.x < QBLK ? ahead_g : ahead_u;
    const Blocks& scale_of = threadIdx.x < QBLK ? P.gate : P.up;
    const int scale_row = threadIdx.x & (QBLK - 1);
    const bool brings = threadIdx.x < 2 * QBLK;
    clear_maxima(S);
    TilePos p = tile_at(blockIdx.x, P.tiles_c, rows, cols, P.vec);
    fetch(p, 0);
    if (brings && p.full) coded_scales(scale_slot, 0)[scale_row] = fetch_scale(scale_of, p, scale_row);
#pragma unroll 1
    for (uint32_t tile = blockIdx.x; tile < P.tiles; par ^= 1) {
        float v[3][R][8];                // read as dh, g, u
        cp_async_wait();
        __syncthreads();                 // everybody's pieces have landed, the last tile's shared words have been read
        read_matrix<T>(ahead_dh, (const T*)P.dh, P.ld_dh, rows, cols, P.vec, p, v[0]);
        read_coded(ahead_g, par, P.gate, rows, cols, p, v[1]);
        read_coded(ahead_u, par, P.up, rows, cols, p, v[2]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                auto two = [&](int m) { return make_float2(v[m][i][j], v[m][i][j + 1]); };
                auto put = [&](int m, float2 x) { v[m][i][j] = x.x; v[m][i][j + 1] = x.y; };
                const float2 dh = two(0), g = two(1), u = two(2), one = make_float2(1.0f, 1.0f), minus = make_float2(-1.0f, -1.0f);
                float2 dz;
                const float2 pr = logistic2<GELU>(g, &dz), a = __fmul2_rn(g, pr);
                float2 tail = __fmul2_rn(a, __ffma2_rn(pr, minus, one));
                if constexpr (GELU) tail = __fmul2_rn(tail, dz);
                put(0, __fmul2_rn(__fmul2_rn(dh, u), __fadd2_rn(tail, pr)));
                put(1, __fmul2_rn(dh, a));
                put(2, __fmul2_rn(a, u));
            }
        }
        const uint32_t next_tile = tile + gridDim.x;
        const TilePos np = tile_at(next_tile < P.tiles ? next_tile : tile, P.tiles_c, rows, cols, P.vec);
        float next_scale = 0.0f;
        auto next = [&] {
            if (sizeof(T) == 4) __syncthreads();
            if (next_tile >= P.tiles) return;
            fetch(np, par ^ 1);
            if (brings && np.full) next_scale = fetch_scale(scale_of, np, scale_row);
        };
        if (p.full) emit_tile<3, SR, true>(v, P.out, p, par, S, later, next);
        else emit_tile<3, SR, false>(v, P.out, p, par, S, later, next);
        if (brings) coded_scales(scale_slot, par ^ 1)[scale_row] = next_scale;
        tile = next_tile;
        p = np;
    }
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static uint32_t tiles_of(int64_t rows, int64_t cols) { return (uint32_t)(((rows + QBLK - 1) / QBLK) * ((cols + QBLK - 1) / QBLK)); }

// SM count of the current device, and the one-time opt-in to more than 48 KB of shared memory.
template <typename K>
static bool prepare_kernel(K kernel, int smem) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess; }
template <typename T>
constexpr int glu_bwd_smem() { return (int)(sizeof(TileShared<3>) + 15) / 16 * 16 + matrix_slot<T>() + 2 * coded_slot(); }

template <typename T>
static bool prepare_glu() {
    const int n = glu_bwd_smem<T>();
    return prepare_kernel(glu_bwd_kernel<T, false, false>, n) && prepare_kernel(glu_bwd_kernel<T, false, true>, n) &&
           prepare_kernel(glu_bwd_kernel<T, true, false>, n) && prepare_kernel(glu_bwd_kernel<T, true, true>, n);
}
static int tile_device() {
    static int sms[64] = {};
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    std::lock_guard<std::mutex> lock(mu);
    if (sms[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 0;
        if (!prepare_kernel(quantize_blocks_kernel<0, false>, matrix_slot<float>()) || !prepare_kernel(quantize_blocks_kernel<0, true>, matrix_slot<float>()) ||
            !prepare_kernel(quantize_blocks_kernel<1, false>, matrix_slot<__nv_bfloat16>()) || !prepare_kernel(quantize_blocks_kernel<1, true>, matrix_slot<__nv_bfloat16>()) ||
            !prepare_kernel(quantize_blocks_kernel<2, false>, coded_slot()) || !prepare_kernel(quantize_blocks_kernel<2, true>, coded_slot()) ||
            !prepare_glu<float>() || !prepare_glu<__nv_bfloat16>())
            return 0;
        sms[dev] = n;
    }
    return sms[dev];
}
// Persistent CTAs, at most as many as are resident at a time.  CTA i takes tiles i, i + grid, ...: the CTAs with one tile
// more than the others come first and land on different SMs.
static unsigned persistent_grid(uint32_t tiles, uint32_t resident) { return tiles < resident ? tiles : resident; }

cudaError_t launch_quantize_blocks(const BlockSource& src, const BlockRounding& rnd, const Blocks& rm, const Blocks& tr,
                                   uint32_t* status, cudaStream_t stream) {
    const int sms = tile_device();
    if (sms == 0) return cudaErrorUnknown;
    QuantBlocksParams P;
    P.src = src;
    P.out.rm[0] = rm; P.out.tr[0] = tr; P.out.rows = src.rows; P.out.cols = src.cols;
    P.out.index_offset = rnd.index_offset; P.out.keys[0] = make_philox_keys(rnd.seed, rnd.tensor_id); P.out.step = rnd.step;
    P.out.status = status;
    P.tiles = tiles_of(src.rows, src.cols); P.tiles_c = (uint32_t)((src.cols + QBLK - 1) / QBLK);
    P.vec = src.coded.codes ? 1 : (uintptr_t)src.x % 16 == 0 && src.ld % (src.dt == SRQ_F32 ? 4 : 8) == 0;
    const dim3 grid(persistent_grid(P.tiles, (uint32_t)sms * (rnd.sr ? 1 : 2))), block(TQ_THREADS);
    cudaError_t e;
    if (src.coded.codes)
        e = rnd.sr ? launch_pdl(quantize_blocks_kernel<2, true>, grid, block, coded_slot(), stream, P) : launch_pdl(quantize_blocks_kernel<2, false>, grid, block, coded_slot(), stream, P);
    else if (src.dt == SRQ_BF16)
        e = rnd.sr ? launch_pdl(quantize_blocks_kernel<1, true>, grid, block, matrix_slot<__nv_bfloat16>(), stream, P)
                   : launch_pdl(quantize_blocks_kernel<1, false>, grid, block, matrix_slot<__nv_bfloat16>(), stream, P);
    else
        e = rnd.sr ? launch_pdl(quantize_blocks_kernel<0, true>, grid, block, matrix_slot<float>(), stream, P)
                   : launch_pdl(quantize_blocks_kernel<0, false>, grid, block, matrix_slot<float>(), stream, P);
    count_launch();
    return e;
}

template <typename T>
static cudaError_t launch_glu_bwd_t(const GluBwdParams& P, int32_t act, int sr, dim3 grid, cudaStream_t stream) {
    const dim3 block(TQ_THREADS);
    const size_t smem = glu_bwd_smem<T>();
    if (act == SRQ_GELU) return sr ? launch_pdl(glu_bwd_kernel<T, true, true>, grid, block, smem, stream, P) : launch_pdl(glu_bwd_kernel<T, true, false>, grid, block, smem, stream, P);
    return sr ? launch_pdl(glu_bwd_kernel<T, false, true>, grid, block, smem, stream, P) : launch_pdl(glu_bwd_kernel<T, false, false>, grid, block, smem, stream, P);
}

cudaError_t launch_glu_bwd(const void* dh, int32_t dt, int64_t ld_dh, const Blocks& gate, const Blocks& up, int64_t T, int64_t F,
                           int32_t act, const BlockRounding& rnd, const Blocks& dg, const Blocks& du, const Blocks& dg_t,
                           const Blocks& du_t, const Blocks& h_t, uint32_t* status, cudaStream_t stream) {
    const int sms = tile_device();
    if (sms == 0) return cudaErrorUnknown;
    GluBwdParams P;
    P.dh = dh; P.ld_dh = ld_dh; P.gate = gate; P.up = up;
    P.out.rm[0] = dg; P.out.rm[1] = du; P.out.tr[0] = dg_t; P.out.tr[1] = du_t; P.out.tr[2] = h_t;
    P.out.rows = T; P.out.cols = F; P.out.index_offset = rnd.index_offset; P.out.step = rnd.step; P.out.status = status;
    for (int i = 0; i < 3; ++i) P.out.keys[i] = make_philox_keys(rnd.seed, rnd.tensor_id + (uint64_t)i);
    P.tiles = tiles_of(T, F); P.tiles_c = (uint32_t)((F + QBLK - 1) / QBLK);
    P.vec = (uintptr_t)dh % 16 == 0 && ld_dh % (dt == SRQ_F32 ? 4 : 8) == 0;
    const dim3 grid(persistent_grid(P.tiles, (uint32_t)sms));
    const cudaError_t e = dt == SRQ_F32 ? launch_glu_bwd_t<float>(P, act, rnd.sr, grid, stream) : launch_glu_bwd_t<__nv_bfloat16>(P, act, rnd.sr, grid, stream);
    count_launch();
    return e;
}

}  // namespace srq
