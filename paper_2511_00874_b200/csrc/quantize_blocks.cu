// Block-scaled E4M3 quantizer (1 x 128 blocks or 128 x 128 tiles, row-major and / or transposed) and the
// backward pass of the gated feed-forward block, which is the same kernel over values it computes itself.
//
// One CTA of 512 threads per 128 x 128 tile.  Thread (g, l), g = 0..31, l = 0..15, holds rows 4 g .. 4 g + 3 of
// columns 8 l .. 8 l + 7 in registers, so that
//   - a row's 128 values sit in 16 neighbouring lanes: its absmax is four shuffles;
//   - a column's 128 values sit in 32 threads of 16 warps: its absmax is one shuffle and one shared atomic;
//   - the transposed codes of a thread are 8 words of 4 bytes, which meet in a swizzled shared tile.
// The tile is read once whatever is written: both layouts and both kinds of step size come from the registers.
// Bound by HBM.
#include "blocks.cuh"

namespace srq {

constexpr int TQ_THREADS = 512;

struct TileShared {
    uint32_t col_max[QBLK];          // [column % 8][column / 8]: a warp's atomics hit 16 different banks
    float col_inv[QBLK];             // same order
    uint32_t tile_max;
    uint32_t words[QBLK * 32];       // transposed codes: column c's rows 4 g .. 4 g + 3 at [c][g ^ 2 (c / 8)]
};

struct TilePos {
    int64_t r0, c0, rows, cols;      // tile origin, extents of the matrix
    int g, l;                        // row quad and column octet of the thread
};

// Quantizes the tile held as v (zeros outside the matrix) into rm and / or tr.  rnd: thresholds (SR only).
// All threads of the CTA call it together.
template <bool SR>
__device__ __forceinline__ void emit_tile(const float (&v)[4][8], const uint32_t (&rnd)[SR ? 4 : 1][8], const Blocks& rm,
                                          const Blocks& tr, const TilePos& p, TileShared* S, uint32_t* status) {
    const int tid = threadIdx.x, lane = tid & 31;
    const bool want_rm = rm.codes != nullptr, want_tr = tr.codes != nullptr;
    const bool tile_rm = want_rm && rm.tile_rows > 1, tile_tr = want_tr && tr.tile_rows > 1;
    uint32_t row_max[4] = {0u, 0u, 0u, 0u};
    if (want_rm || tile_tr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row_max[i] = abs_word(absmax3(absmax3(v[i][0], v[i][1], v[i][2]), absmax3(v[i][3], v[i][4], v[i][5]), absmax3(v[i][6], v[i][7], 0.0f)));
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) row_max[i] = max(row_max[i], __shfl_xor_sync(0xFFFFFFFFu, row_max[i], s));
        }
    }
    if (want_tr || tile_rm) {        // the CTA has to meet
        if (tid < QBLK) S->col_max[tid] = 0u;
        if (tid == 0) S->tile_max = 0u;
        __syncthreads();
        if (tile_rm || tile_tr) {
            uint32_t m = max(max(row_max[0], row_max[1]), max(row_max[2], row_max[3]));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
            if (lane == 0) atomicMax(&S->tile_max, m);
        }
        if (want_tr && !tile_tr) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t m = abs_word(absmax3(absmax3(v[0][j], v[1][j], v[2][j]), v[3][j], 0.0f));
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                if (lane < 16) atomicMax(&S->col_max[j * 16 + p.l], m);
            }
        }
        __syncthreads();
        if (want_tr && tid < QBLK) {
            const int64_t c = p.c0 + (tid & 15) * 8 + (tid >> 4);
            const uint32_t m = tile_tr ? S->tile_max : S->col_max[tid];
            float step, inv;
            block_step(m, &step, &inv);
            S->col_inv[tid] = inv;
            if (block_nonfinite(m)) note(status, SRQ_ERR_NONFINITE);
            if (!tile_tr && c < p.cols) tr.scale[c * tr.ld_scale + p.r0 / QBLK] = step;
            if (tile_tr && tid == 0) tr.scale[(p.c0 / QBLK) * tr.ld_scale + p.r0 / QBLK] = step;
        }
    }
    if (want_rm) {
        // the divisions of four rows once per thread: lane l of a row's sixteen does row l % 4's
        const int pick = p.l & 3;
        uint32_t m = pick == 0 ? row_max[0] : pick == 1 ? row_max[1] : pick == 2 ? row_max[2] : row_max[3];
        if (tile_rm) m = S->tile_max;
        float step, inv;
        block_step(m, &step, &inv);
        if (block_nonfinite(m)) note(status, SRQ_ERR_NONFINITE);
        const int64_t r_mine = p.r0 + 4 * p.g + pick;
        if (!tile_rm && p.l < 4 && r_mine < p.rows) rm.scale[r_mine * rm.ld_scale + p.c0 / QBLK] = step;
        if (tile_rm && tid == 0) rm.scale[(p.r0 / QBLK) * rm.ld_scale + p.c0 / QBLK] = step;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __shfl_sync(0xFFFFFFFFu, inv, (lane & 16) + i);
            const int64_t r = p.r0 + 4 * p.g + i, c = p.c0 + 8 * p.l;
            uint32_t w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                w[h] = encode4<SR>(v[i][4 * h], v[i][4 * h + 1], v[i][4 * h + 2], v[i][4 * h + 3], f, f, f, f,
                                   rnd[SR ? i : 0][4 * h], rnd[SR ? i : 0][4 * h + 1], rnd[SR ? i : 0][4 * h + 2], rnd[SR ? i : 0][4 * h + 3]);
            if (r < p.rows && c < p.cols) store_codes8(rm.codes + r * rm.ld, c, p.cols, w[0], w[1]);
        }
    }
    if (want_tr) {
        __syncthreads();             // reciprocals are there
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = S->col_inv[j * 16 + p.l];
            S->words[(8 * p.l + j) * 32 + (p.g ^ (2 * p.l))] =
                encode4<SR>(v[0][j], v[1][j], v[2][j], v[3][j], f, f, f, f, rnd[0][j], rnd[SR ? 1 : 0][j], rnd[SR ? 2 : 0][j], rnd[SR ? 3 : 0][j]);
        }
        __syncthreads();
        const int warp = tid >> 5;
        const int64_t r = p.r0 + 4 * lane;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int cc = 8 * warp + k;
            const int64_t c = p.c0 + cc;
            if (c >= p.cols || r >= p.rows) continue;
            const uint32_t w = S->words[cc * 32 + (lane ^ (2 * warp))];
            uint8_t* dst = tr.codes + c * tr.ld + r;
            if (r + 4 <= p.rows) *reinterpret_cast<uint32_t*>(dst) = w;
            else
                for (int e = 0; e < 4 && r + e < p.rows; ++e) dst[e] = (uint8_t)(w >> (8 * e));
        }
    }
}

__device__ __forceinline__ TilePos tile_pos(int64_t rows, int64_t cols) {
    const int64_t n_tc = (cols + QBLK - 1) / QBLK;
    TilePos p;
    p.r0 = (int64_t)blockIdx.x / n_tc * QBLK;
    p.c0 = (int64_t)blockIdx.x % n_tc * QBLK;
    p.rows = rows; p.cols = cols;
    p.l = threadIdx.x & 15; p.g = threadIdx.x >> 4;
    return p;
}

// Eight consecutive numbers of a block-coded row (c a multiple of 8; columns >= cols read as 0).
__device__ __forceinline__ void load_coded8(const Blocks& b, int64_t r, int64_t c, int64_t cols, float v[8]) {
    const uint8_t* row = b.codes + r * b.ld;
    uint2 w = make_uint2(0u, 0u);
    if (c + 8 <= cols) {
        w = *reinterpret_cast<const uint2*>(row + c);
    } else {
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) (e < 4 ? w.x : w.y) |= (uint32_t)row[c + e] << (8 * (e & 3));
    }
    const float s = c < cols ? b.scale[(b.tile_rows > 1 ? r / QBLK : r) * b.ld_scale + c / QBLK] : 0.0f;
    e4m3x4_to_f32(w.x, v);
    e4m3x4_to_f32(w.y, v + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], s);
}

struct QuantBlocksParams {
    BlockSource src;
    Blocks rm, tr;
    uint64_t index_offset;
    PhiloxKeys keys;
    int32_t vec;                     // 16-byte loads of the source allowed
    uint32_t* status;
};

// SRC: 0 binary32, 1 bfloat16, 2 block codes.
template <int SRC, bool SR>
__global__ void __launch_bounds__(TQ_THREADS, SR ? 1 : 2) quantize_blocks_kernel(const __grid_constant__ QuantBlocksParams P) {
    pdl_enter();
    __shared__ TileShared S;
    const TilePos p = tile_pos(P.src.rows, P.src.cols);
    float v[4][8];
    uint32_t rnd[SR ? 4 : 1][8] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = p.r0 + 4 * p.g + i, c = p.c0 + 8 * p.l;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        if (r < p.rows) {
            if constexpr (SRC == 0) load8((const float*)P.src.x + r * P.src.ld, c, p.cols, P.vec, v[i]);
            else if constexpr (SRC == 1) load8((const __nv_bfloat16*)P.src.x + r * P.src.ld, c, p.cols, P.vec, v[i]);
            else load_coded8(P.src.coded, r, c, p.cols, v[i]);
        }
        if constexpr (SR) thresholds8(P.index_offset + (uint64_t)r * (uint64_t)p.cols + (uint64_t)c, P.keys, rnd[i]);
    }
    emit_tile<SR>(v, rnd, P.rm, P.tr, p, &S, P.status);
}

struct GluBwdParams {
    const void* dh; int64_t ld_dh;
    Blocks gate, up, dg, du, dg_t, du_t, h_t;
    int64_t T, F;
    uint64_t index_offset;
    PhiloxKeys keys[3];              // of dg, du, h
    int32_t vec;
    uint32_t* status;
};

// dg = dh u act'(g), du = dh act(g), h = act(g) u over one tile, each quantized as it is formed.  dh and
// the codes of g and u stay in registers; the activation is evaluated anew for each of the three.
template <typename T, bool GELU, bool SR>
__global__ void __launch_bounds__(TQ_THREADS, 1) glu_bwd_kernel(const __grid_constant__ GluBwdParams P) {
    pdl_enter();
    __shared__ TileShared S;
    const TilePos p = tile_pos(P.T, P.F);
    float dh[4][8], g[4][8], u[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = p.r0 + 4 * p.g + i, c = p.c0 + 8 * p.l;
#pragma unroll
        for (int j = 0; j < 8; ++j) dh[i][j] = g[i][j] = u[i][j] = 0.0f;
        if (r < p.rows) {
            if (P.dh) load8((const T*)P.dh + r * P.ld_dh, c, p.cols, P.vec, dh[i]);
            load_coded8(P.gate, r, c, p.cols, g[i]);
            load_coded8(P.up, r, c, p.cols, u[i]);
        }
    }
    const Blocks none;
#pragma unroll 1
    for (int which = 0; which < 3; ++which) {
        const Blocks& rm = which == 0 ? P.dg : which == 1 ? P.du : none;
        const Blocks& tr = which == 0 ? P.dg_t : which == 1 ? P.du_t : P.h_t;
        if (!rm.codes && !tr.codes) continue;
        float v[4][8];
        uint32_t rnd[SR ? 4 : 1][8] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float dz;
                const float pr = logistic_of<GELU>(g[i][j], &dz), a = g[i][j] * pr;
                v[i][j] = which == 0 ? dh[i][j] * u[i][j] * fmaf(a * (1.0f - pr), dz, pr) : which == 1 ? dh[i][j] * a : a * u[i][j];
            }
            if constexpr (SR)
                thresholds8(P.index_offset + (uint64_t)(p.r0 + 4 * p.g + i) * (uint64_t)p.cols + (uint64_t)(p.c0 + 8 * p.l), P.keys[which], rnd[i]);
        }
        emit_tile<SR>(v, rnd, rm, tr, p, &S, P.status);
    }
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static int64_t tiles_of(int64_t rows, int64_t cols) { return ((rows + QBLK - 1) / QBLK) * ((cols + QBLK - 1) / QBLK); }

cudaError_t launch_quantize_blocks(const BlockSource& src, const BlockRounding& rnd, const Blocks& rm, const Blocks& tr,
                                   uint32_t* status, cudaStream_t stream) {
    QuantBlocksParams P;
    P.src = src; P.rm = rm; P.tr = tr; P.index_offset = rnd.index_offset;
    P.keys = make_philox_keys(rnd.seed, rnd.tensor_id);
    const int per16 = src.dt == SRQ_F32 ? 4 : 8;
    P.vec = src.x && (uintptr_t)src.x % 16 == 0 && src.ld % per16 == 0;
    P.status = status;
    const dim3 grid((unsigned)tiles_of(src.rows, src.cols)), block(TQ_THREADS);
    cudaError_t e;
    if (src.coded.codes) e = rnd.sr ? launch_pdl(quantize_blocks_kernel<2, true>, grid, block, 0, stream, P) : launch_pdl(quantize_blocks_kernel<2, false>, grid, block, 0, stream, P);
    else if (src.dt == SRQ_BF16) e = rnd.sr ? launch_pdl(quantize_blocks_kernel<1, true>, grid, block, 0, stream, P) : launch_pdl(quantize_blocks_kernel<1, false>, grid, block, 0, stream, P);
    else e = rnd.sr ? launch_pdl(quantize_blocks_kernel<0, true>, grid, block, 0, stream, P) : launch_pdl(quantize_blocks_kernel<0, false>, grid, block, 0, stream, P);
    count_launch();
    return e;
}

template <typename T>
static cudaError_t launch_glu_bwd_t(const GluBwdParams& P, int32_t act, int sr, dim3 grid, cudaStream_t stream) {
    const dim3 block(TQ_THREADS);
    if (act == SRQ_GELU) return sr ? launch_pdl(glu_bwd_kernel<T, true, true>, grid, block, 0, stream, P) : launch_pdl(glu_bwd_kernel<T, true, false>, grid, block, 0, stream, P);
    return sr ? launch_pdl(glu_bwd_kernel<T, false, true>, grid, block, 0, stream, P) : launch_pdl(glu_bwd_kernel<T, false, false>, grid, block, 0, stream, P);
}

cudaError_t launch_glu_bwd(const void* dh, int32_t dt, int64_t ld_dh, const Blocks& gate, const Blocks& up, int64_t T, int64_t F,
                           int32_t act, const BlockRounding& rnd, const Blocks& dg, const Blocks& du, const Blocks& dg_t,
                           const Blocks& du_t, const Blocks& h_t, uint32_t* status, cudaStream_t stream) {
    GluBwdParams P;
    P.dh = dh; P.ld_dh = ld_dh; P.gate = gate; P.up = up;
    P.dg = dg; P.du = du; P.dg_t = dg_t; P.du_t = du_t; P.h_t = h_t;
    P.T = T; P.F = F; P.index_offset = rnd.index_offset;
    for (int i = 0; i < 3; ++i) P.keys[i] = make_philox_keys(rnd.seed, rnd.tensor_id + (uint64_t)i);
    P.vec = (uintptr_t)dh % 16 == 0 && ld_dh % (dt == SRQ_F32 ? 4 : 8) == 0;
    P.status = status;
    const dim3 grid((unsigned)tiles_of(T, F));
    const cudaError_t e = dt == SRQ_F32 ? launch_glu_bwd_t<float>(P, act, rnd.sr, grid, stream) : launch_glu_bwd_t<__nv_bfloat16>(P, act, rnd.sr, grid, stream);
    count_launch();
    return e;
}

}  // namespace srq
