// Products of block-coded E4M3 matrices on the 5th-generation tensor cores, and the gated feed-forward block
// as an epilogue of the same kernels.
//
//   out[i, j] = sum_k sA[i, k] sB[j, k] P_k[i, j],     P_k = the 128-long piece k of the contraction
//
// The step sizes change every 128 values of the contraction, so the tensor core cannot add up the whole sum:
// each P_k is left in TMEM for itself (kind::f8f6f4, binary32), read back and added into binary32 registers
// with its factor.  That takes one tcgen05.ld and one multiply-add per element and k-block (two where every row and
// every column has a step size of its own), next to the 512 cycles the MMAs of a 128 x 256 x 128 piece take: the two run
// side by side, k-block by k-block, through two TMEM buffers.
//
// gemm_blocks_kernel: 256 x 256 tiles on CTA pairs (tcgen05.mma.cta_group::2), persistent.
//   warp 0      TMA producer (128-byte swizzled tiles, ring of 5 stages of 32 KB)
//   warp 1      TMEM and MMA issue (leader CTA): a k-block goes into one TMEM buffer as two M256 N128 halves with barriers
//               of their own, so that the first half's sums are added up while the second is multiplied
//   warps 2-3   step sizes: four k-blocks at a time from global memory into a shared ring, so that the warps that
//               add up hold no addresses and no prefetched values in their registers
//   warps 4-19  four groups of four; a thread owns one row of the CTA's 128 and 64 of the 256 columns: group g columns
//               64 g .. in a plain product; in the gated block, whose 256 columns are 128 of the gate and 128 of the up
//               projection (one CTA of the pair stages Wg, the other Wu), columns 32 g .. 32 g + 31 of both, so that
//               g and u of an element meet in one thread
// Measured, by machine and clock: 16384 x 4096 x 4096, 128 x 128 tiles on b, 257 to 300 us (2.1 to 1.8 PFLOP/s); 5632 x 2048 x
// 8192, 1 x 128 on both, 150 to 169 us, 95 to 117 with tiles on b, 178 accumulating; gated 16384 x 2048 x 5632 with checkpoints
// 453 to 515 us.  No pipe is at its limit (tensor 56 % of the cycles, issue 58 %): the MMAs, the reads of their sums and the
// additions wait for one another.  Eight adding warps with 128 sums each: 322 us for the first; a second issuing warp, and
// 16 columns read while 16 are added: no difference.
//
// gemm_blocks_small_kernel: few tokens.  The roles turn around: 128 rows of the weights are the M of the MMA and
// 16 to 128 tokens its N, the contraction is cut over a cluster of CTAs (as many as fill the machine), and the
// parts are added through distributed shared memory in a fixed order.  Reading the weights once is all there
// is to do, and every SM reads its share with up to 200 KB in flight.  Warp 0 loads, warp 1 issues, four or eight warps
// scale and add up.  1 x 4096 x 4096: 6.8 us, of which 2.6 are the weights at the copy rate.
//
// Every wait is bounded (2 s); on expiry SRQ_ERR_TIMEOUT is recorded, all roles run to their end without
// waiting any more, and TMEM is freed.
#include <cuda.h>

#include <climits>
#include <mutex>
#include <type_traits>

#include "blocks.cuh"
#include "tensor_core.cuh"

namespace srq {

constexpr int GB_M = 128, GB_N = 256, GB_K = 128;      // rows per CTA, tile columns, bytes (= codes) per k-block
constexpr int GB_STAGES = 5;
constexpr int GB_STAGE_BYTES = GB_M * GB_K + (GB_N / 2) * GB_K;
constexpr int GB_ADD_WARPS = 16;                       // warps that read TMEM, scale, add up and store
constexpr int GB_CGROUPS = GB_ADD_WARPS / 4;           // column groups of the tile; a thread holds one row of one group
constexpr int GB_COLS = GB_N / GB_CGROUPS;             // sums per thread
constexpr int GB_THREADS = 128 + 32 * GB_ADD_WARPS;
// Registers: 640 threads start with 96 each; the first warpgroup keeps 32 and the four that hold 64 sums per thread
// take 112 (32 + 4 x 112 = 5 x 96: exactly what the block was launched with).
constexpr int GB_REGS_FEW = 32, GB_REGS_MANY = 112;
constexpr int GB_OUT_BYTES = 32 * 64;                  // staging block of an epilogue warp: 32 rows of 64 bytes
constexpr int GB_UMMA_K = 32;
constexpr int GB_SCALE_SLOTS = 3;                      // chunks of four k-blocks whose step sizes are in shared memory

struct GemmBlocksParams {
    int64_t M, N;                       // N: columns of out, or of h (the gated block's F)
    int32_t num_kb, tiles_m, tiles_n;
    int32_t full_tiles, half_kb;        // pairs: tiles from full_tiles on are done in two parts, k-blocks [0, half_kb) and the rest
    Blocks a, b, b2;                    // b2: up projection of the gated block
    int32_t a_vec, b_vec;               // 16-byte loads of four step sizes allowed
    void* out; int64_t ldo; int32_t out_bf16, tma_out, accumulate;
    Blocks h, gate, up;                 // gated block
    int32_t gelu, h_vec;
    uint32_t* status;
};

struct GbTail {
    uint64_t full[GB_STAGES], empty[GB_STAGES], tmem_full[2][2], tmem_empty[2][2], drain;     // [half][buffer]
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    uint64_t scale_full[GB_SCALE_SLOTS], scale_empty[GB_SCALE_SLOTS];
    alignas(16) float row_scale[GB_SCALE_SLOTS][4][GB_M];   // [slot][k-block of the chunk][row]
    alignas(16) float col_scale[GB_SCALE_SLOTS][4][GB_N];   // [..][column of the tile], or [0], [1]: one per 128 columns
    uint32_t amax[2][3][GB_CGROUPS][GB_M];         // gated block: [tile parity][h, gate, up][column group][row]
    float inv[2][3][GB_M];
};
constexpr size_t gb_smem() { return 1024 + (size_t)GB_STAGES * GB_STAGE_BYTES + GB_ADD_WARPS * GB_OUT_BYTES + sizeof(GbTail); }

__device__ __forceinline__ void gb_give_up(volatile uint32_t* abort_flag, uint32_t* status) {
    *abort_flag = 1u;
    note(status, SRQ_ERR_TIMEOUT);
}

__device__ __forceinline__ uint32_t elect_one() {
    uint32_t e;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e;
}

// Bounded wait of the warps that add up, on a barrier's shared address.  The usual case is one try; when the limit has
// passed or another role has given up it returns all the same, so that the caller needs no second path: its
// results are then garbage, the status says so, and every wait after it returns as soon.
// The lanes may leave the loop at different times; they meet before they return, because a tcgen05.ld.sync.aligned follows.
__device__ __forceinline__ bool try_wait_addr(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void wait_or_abort(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status) {
    if (!try_wait_addr(bar, parity)) {
        const uint64_t t0 = global_ns();
        while (!try_wait_addr(bar, parity)) {
            if (*abort_flag) break;
            if (global_ns() - t0 > WAIT_LIMIT_NS) { gb_give_up(abort_flag, status); break; }
        }
    }
    __syncwarp();
}

// Bounded wait of a whole warp, with one vote: the usual case is that the phase has completed.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint64_t* b, volatile uint32_t* abort_flag) {
    if (__all_sync(0xFFFFFFFFu, try_wait_addr(bar, parity))) return true;
    return __all_sync(0xFFFFFFFFu, mbar_wait(b, parity, abort_flag));
}

// 32 lanes x 16 columns of TMEM (in registers after tmem_ld_wait).
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
// Step sizes of k-blocks 4 c .. 4 c + 3 of one scale row (zeros past num_kb).  Ordinary loads: the kernel may have been launched
// while its predecessor was still writing them, and the read-only path is for data that nobody writes while a kernel runs.
__device__ __forceinline__ float4 scales4(const float* row, int32_t c, int32_t num_kb, bool vec) {
    const int32_t k = 4 * c;
    if (row == nullptr || k >= num_kb) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (vec && k + 4 <= num_kb) return *reinterpret_cast<const float4*>(row + k);
    float4 f = make_float4(row[k], 0.0f, 0.0f, 0.0f);
    if (k + 1 < num_kb) f.y = row[k + 1];
    if (k + 2 < num_kb) f.z = row[k + 2];
    if (k + 3 < num_kb) f.w = row[k + 3];
    return f;
}
__device__ __forceinline__ float pick4(const float4& f, int32_t i) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; }

__device__ __forceinline__ float2 pair(uint32_t a, uint32_t b) { return make_float2(__uint_as_float(a), __uint_as_float(b)); }

// 4 W consecutive codes of a row from column c (rows start on 16-byte boundaries, c is a multiple of 16).
template <int W>
__device__ __forceinline__ void store_codes(uint8_t* row, int64_t c, int64_t cols, const uint32_t (&w)[W]) {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
        if (c + 16 * q + 16 <= cols) {
            *reinterpret_cast<uint4*>(row + c + 16 * q) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c + 16 * q + e < cols) row[c + 16 * q + e] = (uint8_t)(w[4 * q + (e >> 2)] >> (8 * (e & 3)));
        }
    }
}

// The same for 32 bytes per row in the 32-byte swizzle (16-byte chunk index xor row / 4 mod 2).
__device__ __forceinline__ void stage_rows32(uint32_t stage, int lane, const uint32_t (&w)[8]) {
    const uint32_t row = stage + (uint32_t)lane * 32u;
#pragma unroll
    for (int q = 0; q < 2; ++q)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + (uint32_t)((q ^ ((lane >> 2) & 1)) << 4)),
                     "r"(w[4 * q]), "r"(w[4 * q + 1]), "r"(w[4 * q + 2]), "r"(w[4 * q + 3]) : "memory");
}
// Thread `lane` holds 64 bytes of row `lane` of a block of 32 rows: writes them in the 64-byte swizzle of the output's
// tensor map (16-byte chunk index xor row / 2 mod 4), which also spreads the 16-byte stores of a warp over all banks.
__device__ __forceinline__ void stage_rows64(uint32_t stage, int lane, const uint32_t (&w)[16]) {
    const uint32_t row = stage + (uint32_t)lane * 64u;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + (uint32_t)((q ^ ((lane >> 1) & 3)) << 4)),
                     "r"(w[4 * q]), "r"(w[4 * q + 1]), "r"(w[4 * q + 2]), "r"(w[4 * q + 3]) : "memory");
}

// map_out: of out, or of h's codes.  GLU: the gated block's epilogue instead of the plain one.  COLV: b has a step size per
// row (per column of out), not per 128 of them.
template <bool GLU, bool COLV>
__global__ void __launch_bounds__(GB_THREADS, 1)
gemm_blocks_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_b2, const __grid_constant__ CUtensorMap map_out,
                   const __grid_constant__ CUtensorMap map_gate, const __grid_constant__ CUtensorMap map_up,
                   const __grid_constant__ GemmBlocksParams P) {
    pdl_trigger();                       // the wait follows the set-up below, which touches only shared memory and TMEM
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* out_stage = smem + (size_t)GB_STAGES * GB_STAGE_BYTES;
    GbTail* T = (GbTail*)(out_stage + GB_ADD_WARPS * GB_OUT_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < GB_STAGES; ++s) { mbar_init(&T->full[s], 1); mbar_init(&T->empty[s], 1); }
        for (int b = 0; b < 4; ++b) { mbar_init(&T->tmem_full[0][b], 1); mbar_init(&T->tmem_empty[0][b], GB_ADD_WARPS); }   // half of the warps of both CTAs
        for (int b = 0; b < GB_SCALE_SLOTS; ++b) { mbar_init(&T->scale_full[b], 64); mbar_init(&T->scale_empty[b], GB_ADD_WARPS); }
        mbar_init(&T->drain, 1);
        T->abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<2>(&T->tmem_base, 512);
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    // All 512 columns are this CTA's, so they start at 0: as a constant the address needs no move into a uniform register
    // before every MMA (40 cycles each).
    constexpr uint32_t tmem_base = 0;
    pdl_wait();

    constexpr int TILE_COLS = GLU ? 128 : GB_N;        // columns of the result a tile covers
    // work units: whole tiles, then the halves of the tiles of a last, partly filled round
    const int32_t groups = gridDim.x / 2, group = blockIdx.x / 2;
    const int32_t units = P.full_tiles + 2 * (P.tiles_m * P.tiles_n - P.full_tiles);
    struct Unit { int32_t tm, tn, kb0, kb1; bool half; };
    auto unit = [&](int32_t u) {
        Unit w;
        w.half = !GLU && u >= P.full_tiles;
        const int32_t v = u - P.full_tiles, tile = w.half ? P.full_tiles + (v >> 1) : u;
        w.tm = tile / P.tiles_n; w.tn = tile - w.tm * P.tiles_n;
        w.kb0 = w.half && (v & 1) ? P.half_kb : 0;
        w.kb1 = w.half && !(v & 1) ? P.half_kb : P.num_kb;
        return w;
    };

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(GB_REGS_FEW));
    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            const CUtensorMap* mb = GLU && !leader ? &map_b2 : &map_b;
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(mb) : "memory");
            uint32_t it = 0;
            bool ok = true;
            for (int32_t u = group; u < units && ok; u += groups) {
                const Unit w = unit(u);
                const int32_t tn = w.tn, tm = w.tm;
                const int32_t row_a = (tm * 2 + (int32_t)rank) * GB_M;
                // b's rows so that the first 64 of both CTAs are one half of the tile's columns and the last 64 the other
                const int32_t row_b = GLU ? tn * 128 : tn * GB_N + (int32_t)rank * 64;
                for (int32_t kb = w.kb0; kb < w.kb1; ++kb, ++it) {
                    const uint32_t s = it % GB_STAGES, ph = (it / GB_STAGES) & 1u;
                    if (!mbar_wait(&T->empty[s], ph ^ 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                    if (leader) mbar_expect_tx(&T->full[s], GB_STAGE_BYTES * 2);
                    const uint32_t bar = map_to_cta(smem_u32(&T->full[s]), 0);
                    uint8_t* sa = smem + (size_t)s * GB_STAGE_BYTES;
                    tma_load_2d<2>(sa, &map_a, kb * GB_K, row_a, bar);
                    tma_load_2d<2>(sa + GB_M * GB_K, mb, kb * GB_K, row_b, bar);
                    tma_load_2d<2>(sa + GB_M * GB_K + 64 * GB_K, mb, kb * GB_K, row_b + (GLU ? 64 : 128), bar);
                }
            }
            if (!ok) {
                // loads already issued must land before the CTA may leave
                if (leader) {
                    const uint32_t back = it < (uint32_t)GB_STAGES ? it : (uint32_t)GB_STAGES;
                    for (uint32_t j = 1; j <= back; ++j) {
                        const uint32_t jt = it - j;
                        const uint64_t t0 = global_ns();
                        while (!mbar_try_wait(&T->full[jt % GB_STAGES], (jt / GB_STAGES) & 1u) && global_ns() - t0 < WAIT_LIMIT_NS) {}
                    }
                } else {
                    const uint64_t t0 = global_ns();
                    while (global_ns() - t0 < 1000000ull) {}
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (leader CTA only)
        // The whole warp walks the loop and one elected lane issues: what the instructions take (descriptors, barrier
        // addresses) is then uniform to the compiler and stays in uniform registers.  With a single thread in the loop
        // every MMA cost some 95 cycles and every commit 61 to issue, more than the MMAs themselves take; now the eight MMAs
        // and three commits of a k-block take some 420 together.
        if (leader) {
            constexpr uint32_t idesc = make_idesc(1, GB_M * 2, GB_N / 2);
            const uint32_t elected = elect_one();
            bool ok = true;
            uint32_t s = 0, ph = 0, buf = 0, buf_ph = 1;
            const uint64_t desc0 = make_smem_desc(smem_u32(smem));
            for (int32_t u = group; u < units && ok; u += groups) {
                const Unit w = unit(u);
                for (int32_t kb = w.kb0; kb < w.kb1; ++kb) {
                    ok = warp_wait(smem_u32(&T->full[0]) + 8 * s, ph, &T->full[s], &T->abort_flag);
                    const uint64_t da = desc0 + (uint64_t)(s * (GB_STAGE_BYTES >> 4)), db = da + (uint64_t)((GB_M * GB_K) >> 4);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        ok = ok && warp_wait(smem_u32(&T->tmem_empty[h][0]) + 8 * buf, buf_ph, &T->tmem_empty[h][buf], &T->abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elected) {
#pragma unroll
                            for (int k = 0; k < GB_K / GB_UMMA_K; ++k)
                                umma<2, 1>(tmem_base + buf * GB_N + h * (GB_N / 2), da + (uint64_t)((k * GB_UMMA_K) >> 4),
                                           db + (uint64_t)((h * 64 * GB_K + k * GB_UMMA_K) >> 4), idesc, k ? 1u : 0u);
                            umma_commit<2>(&T->tmem_full[h][buf], true);
                            if (h == 1) umma_commit<2>(&T->empty[s], true);
                        }
                        __syncwarp();
                    }
                    if (!ok) { gb_give_up(&T->abort_flag, P.status); break; }
                    s = s + 1 == (uint32_t)GB_STAGES ? 0u : s + 1;
                    ph ^= s == 0u ? 1u : 0u;
                    buf_ph ^= buf;
                    buf ^= 1u;
                }
            }
            if (!ok && elected) {
                umma_commit<2>(&T->drain, false);
                const uint64_t t0 = global_ns();
                while (!mbar_try_wait(&T->drain, 0u) && global_ns() - t0 < WAIT_LIMIT_NS) {}
            }
        }
    } else {
        // ------------------------------------------------------------------ step sizes (warps 2 and 3)
        // They run up to GB_SCALE_SLOTS chunks ahead, so that the latency of one load after the other does not
        // matter (and their registers are few).
        const int t = threadIdx.x - 64;                  // 0..63: rows t and t + 64, columns t + 64 j
        uint32_t slot = 0, ph = 0;
        bool ok = true;
        auto put = [&](float* dst, int ld, const Blocks& m, int64_t r, int64_t end, int32_t chunk, bool vec) {
            const float* row = r < end ? m.scale + (m.tile_rows > 1 ? r / QBLK : r) * m.ld_scale : nullptr;
            const float4 f = scales4(row, chunk, P.num_kb, vec);
            dst[0] = f.x; dst[ld] = f.y; dst[2 * ld] = f.z; dst[3 * ld] = f.w;
        };
        for (int32_t u = group; u < units && ok; u += groups) {
            const Unit w = unit(u);
            const int64_t row = ((int64_t)w.tm * 2 + rank) * GB_M + t, col = (int64_t)w.tn * TILE_COLS;
            for (int32_t chunk = w.kb0 >> 2; 4 * chunk < w.kb1; ++chunk) {
                if (!mbar_wait(&T->scale_empty[slot], ph ^ 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
#pragma unroll 1
                for (int j = 0; j < 2; ++j) put(&T->row_scale[slot][0][t + 64 * j], GB_M, P.a, row + 64 * j, P.M, chunk, P.a_vec);
                if constexpr (COLV) {
#pragma unroll 1
                    for (int j = 0; j < 4; ++j)
                        put(&T->col_scale[slot][0][t + 64 * j], GB_N, GLU && j >= 2 ? P.b2 : P.b, col + t + 64 * (GLU ? j & 1 : j), P.N, chunk, P.b_vec);
                } else if (t < 2) {
                    put(&T->col_scale[slot][0][t], GB_N, GLU && t == 1 ? P.b2 : P.b, GLU ? col : col + 128 * t, P.N, chunk, P.b_vec);
                }
                mbar_arrive(&T->scale_full[slot]);
                slot = slot + 1 == (uint32_t)GB_SCALE_SLOTS ? 0u : slot + 1;
                ph ^= slot == 0u ? 1u : 0u;
            }
        }
    }
    } else {
        // ------------------------------------------------------------------ scaling and epilogue (warps 4..19)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(GB_REGS_MANY));
        const int quarter = warp & 3, cg = (warp - 4) >> 2;
        const int trow = quarter * 32 + lane;            // row within this CTA's 128
        const uint32_t half = (uint32_t)(GB_COLS * cg / 128);      // of the tile's columns in TMEM: an MMA of its own
        const uint32_t empty0 = map_to_cta(smem_u32(&T->tmem_empty[half][0]), 0);
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
        // first tile column of each of this thread's 32-column pieces: neighbours, or, in the gated block, the same columns
        // of the gate and of the up projection
        constexpr int PIECES = GB_COLS / 32;
        auto piece = [&](int c) -> uint32_t {
            return GLU ? (uint32_t)((c / (PIECES / 2)) * 128 + (GB_COLS / 2) * cg + 32 * (c % (PIECES / 2))) : (uint32_t)(GB_COLS * cg + 32 * c);
        };
        // and where they are in a TMEM buffer: a half holds 128 columns of out, or 64 gate and 64 up columns
        auto column = [&](int c) -> uint32_t { return GLU ? (piece(c) & 64u) * 2u + (piece(c) & 63u) + (piece(c) >> 7) * 64u : piece(c); };
        const uint32_t stage = smem_u32(out_stage + (warp - 4) * GB_OUT_BYTES);
        const uint32_t full0 = smem_u32(&T->tmem_full[half][0]);
        uint32_t buf = 0, buf_ph = 0, par = 0, slot = 0, slot_ph = 0;
        for (int32_t u = group; u < units; u += groups) {
            float2 sum[GB_COLS / 2];                       // two by two
#pragma unroll
            for (int i = 0; i < GB_COLS / 2; ++i) sum[i] = make_float2(0.0f, 0.0f);
#pragma unroll 1
            for (int32_t left = unit(u).kb1 - unit(u).kb0; left > 0; left -= 4) {
                wait_or_abort(smem_u32(&T->scale_full[0]) + 8 * slot, slot_ph, &T->abort_flag, P.status);
                const float* rs = &T->row_scale[slot][0][trow];
                const float* cs = T->col_scale[slot][0];
#pragma unroll 1
                for (int32_t j = min(left, 4); j > 0; --j, rs += GB_M, cs += GB_N) {
                    const float sa = *rs;
                    float2 s0 = make_float2(sa, sa), s1 = s0;
                    if constexpr (!COLV) {
                        const float f0 = __fmul_rn(sa, cs[GLU ? 0 : GB_COLS * cg / 128]);
                        s0 = s1 = make_float2(f0, f0);
                        if constexpr (GLU) { const float f1 = __fmul_rn(sa, cs[1]); s1 = make_float2(f1, f1); }
                    }
                    wait_or_abort(full0 + 8 * buf, buf_ph, &T->abort_flag, P.status);
                    tc_fence_after();
                    const uint32_t tb = taddr + buf * GB_N;
                    // the buffer is handed back as soon as its last piece is in registers
                    auto release = [&]() {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(empty0 + 8 * buf);
                    };
                    if constexpr (!COLV) {
#pragma unroll
                        for (int c = 0; c < PIECES; ++c) {
                            uint32_t v[32];
                            tmem_ld32(tb + column(c), v);
                            tmem_ld_wait();
                            if (c + 1 == PIECES) release();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                sum[16 * c + i] = __ffma2_rn(pair(v[2 * i], v[2 * i + 1]), c < PIECES / 2 ? s0 : s1, sum[16 * c + i]);
                        }
                    } else {
                        // half as many columns at a time: the columns' step sizes take registers too
#pragma unroll
                        for (int c = 0; c < 2 * PIECES; ++c) {
                            uint32_t v[16];
                            tmem_ld16(tb + column(c >> 1) + 16 * (c & 1), v);
                            tmem_ld_wait();
                            if (c + 1 == 2 * PIECES) release();
                            const float* f0 = cs + piece(c >> 1) + 16 * (c & 1);
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float4 f = *reinterpret_cast<const float4*>(f0 + 4 * q);
                                float2& x = sum[8 * c + 2 * q];
                                float2& y = sum[8 * c + 2 * q + 1];
                                x = __ffma2_rn(pair(v[4 * q], v[4 * q + 1]), __fmul2_rn(make_float2(f.x, f.y), s0), x);
                                y = __ffma2_rn(pair(v[4 * q + 2], v[4 * q + 3]), __fmul2_rn(make_float2(f.z, f.w), s0), y);
                            }
                        }
                    }
                    buf_ph ^= buf;
                    buf ^= 1u;
                }
                __syncwarp();                              // this chunk's step sizes have been read
                if (lane == 0) mbar_arrive(&T->scale_empty[slot]);
                slot = slot + 1 == (uint32_t)GB_SCALE_SLOTS ? 0u : slot + 1;
                slot_ph ^= slot == 0u ? 1u : 0u;
            }

            const Unit where = unit(u);
            const int32_t tn = where.tn;
            const int64_t row0 = ((int64_t)where.tm * 2 + rank) * GB_M, row = row0 + trow;
            const int64_t col0 = (int64_t)tn * TILE_COLS;
            float acc[GB_COLS];
#pragma unroll
            for (int i = 0; i < GB_COLS / 2; ++i) { acc[2 * i] = sum[i].x; acc[2 * i + 1] = sum[i].y; }
            if constexpr (GLU) {
                // acc: GH gate columns, then the same GH up columns
                constexpr int GH = GB_COLS / 2;
                static_assert(GH == 32, "a warp's block of codes is 32 x 32");
                const int64_t f0 = col0 + GH * cg;
                const bool live = row < P.M;
                const bool ckpt = P.gate.codes || P.up.codes;
                float h[GH], mg = 0.0f, mu = 0.0f, mh = 0.0f;
                auto gate_all = [&](auto gelu) {
#pragma unroll
                    for (int i = 0; i < GH; i += 2) {
                        const float2 y = gated2<decltype(gelu)::value>(make_float2(acc[i], acc[i + 1]), make_float2(acc[GH + i], acc[GH + i + 1]));
                        h[i] = y.x; h[i + 1] = y.y;
                    }
                };
                if (P.gelu) gate_all(std::true_type()); else gate_all(std::false_type());
#pragma unroll
                for (int i = 0; i < GH; i += 2) mh = absmax3(mh, h[i], h[i + 1]);
                if (ckpt) {
#pragma unroll
                    for (int i = 0; i < GH; i += 2) { mg = absmax3(mg, acc[i], acc[i + 1]); mu = absmax3(mu, acc[GH + i], acc[GH + i + 1]); }
                }
                if (P.out && live) {
                    const bool vec = P.h_vec && f0 + GH <= P.N;
#pragma unroll
                    for (int q = 0; q < GH / 8; ++q) {
                        if (P.out_bf16) store8((__nv_bfloat16*)P.out + row * P.ldo, f0 + 8 * q, P.N, vec, h + 8 * q);
                        else store8((float*)P.out + row * P.ldo, f0 + 8 * q, P.N, vec, h + 8 * q);
                    }
                }
                // a row's 128 columns are in GB_CGROUPS threads: they meet with their maxima, and thread cg of the row does the
                // divisions of matrix cg (h, gate, up) for all of them
                T->amax[par][0][cg][trow] = abs_word(mh);
                if (ckpt) { T->amax[par][1][cg][trow] = abs_word(mg); T->amax[par][2][cg][trow] = abs_word(mu); }
                asm volatile("bar.sync 3, %0;" ::"n"(32 * GB_ADD_WARPS) : "memory");
                float m_mine = 0.0f;
                if (cg < (ckpt ? 3 : 1)) {
                    uint32_t m = 0u;
#pragma unroll
                    for (int i = 0; i < GB_CGROUPS; ++i) m = max(m, T->amax[par][cg][i][trow]);
                    m_mine = __uint_as_float(m);
                    T->inv[par][cg][trow] = block_inv(m);
                }
                asm volatile("bar.sync 3, %0;" ::"n"(32 * GB_ADD_WARPS) : "memory");
                const int32_t wrow = (int32_t)(row0 + quarter * 32);
                auto emit = [&](const Blocks& o, const CUtensorMap* map, int which, uint32_t buffer, const float* val) {
                    if (!o.codes) return;
                    const float inv = T->inv[par][which][trow];
                    uint32_t w[GH / 4];
#pragma unroll
                    for (int q = 0; q < GH / 4; ++q)
                        w[q] = encode4<false>(val[4 * q], val[4 * q + 1], val[4 * q + 2], val[4 * q + 3], inv, inv, inv, inv, 0, 0, 0, 0);
                    if (!P.tma_out) {
                        if (live) store_codes(o.codes + row * o.ld, f0, P.N, w);
                        return;
                    }
                    // 32 rows of 32 codes through shared memory: straight from the registers each store instruction touched 32
                    // lines for 16 bytes each, and a tile's codes took longer than half of its main loop
                    stage_rows32(buffer, lane, w);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0 && wrow < P.M && f0 < P.N) { tma_store_2d(map, buffer, (int32_t)f0, wrow); bulk_commit(); }
                };
                if (lane == 0) bulk_wait_read();         // the last tile's codes have left the two buffers
                __syncwarp();
                if (ckpt) {
                    emit(P.gate, &map_gate, 1, stage, acc);
                    emit(P.up, &map_up, 2, stage + 1024, acc + GH);
                }
                if (cg < (ckpt ? 3 : 1) && live) {
                    const Blocks& o = cg == 0 ? P.h : cg == 1 ? P.gate : P.up;
                    if (o.codes) {
                        if (block_nonfinite(__float_as_uint(m_mine))) note(P.status, SRQ_ERR_NONFINITE);
                        o.scale[row * o.ld_scale + tn] = block_size(__float_as_uint(m_mine));
                    }
                }
                if (P.gate.codes) {
                    // the gate's codes have left the buffer h's take now: all but the newest group, which are the up projection's
                    // where those are wanted, else every group
                    if (lane == 0) {
                        if (P.up.codes) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                        else bulk_wait_read();
                    }
                    __syncwarp();
                }
                emit(P.h, &map_out, 0, stage, h);
                par ^= 1;            // these words are written again two tiles on, a barrier after everyone has read them
            } else {
                const int32_t wrow = (int32_t)(row0 + quarter * 32);
                const int64_t c_first = col0 + GB_COLS * cg;
                // 64 bytes of every row at a time through the warp's staging block, and from there by a block store or, where rows
                // are not aligned for one, row by row with neighbouring lanes on neighbouring columns.  (Straight from the
                // registers every store touched 32 rows: 8191 x 2047 x 300 in bfloat16 169 us, now 25, in binary32 139 and 37.)
                constexpr int F32_BLOCKS = GB_COLS / 16;
                const uint8_t* staged = out_stage + (warp - 4) * GB_OUT_BYTES;
#pragma unroll
                for (int j = 0; j < F32_BLOCKS; ++j) {
                    uint32_t w[16];
                    if (P.out_bf16) {
                        if (j >= F32_BLOCKS / 2) break;
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = j < F32_BLOCKS / 2 ? pack_bf16(acc[(32 * j + 2 * i) % GB_COLS], acc[(32 * j + 2 * i + 1) % GB_COLS]) : 0u;
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(acc[16 * j + i]);
                    }
                    if (P.tma_out && lane == 0) bulk_wait_read();
                    __syncwarp();
                    stage_rows64(stage, lane, w);
                    const int64_t c = c_first + (P.out_bf16 ? 32 : 16) * j;
                    if (P.tma_out) {
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0 && wrow < P.M && c < P.N) {
                            // two halves onto zeros: the same sum in either order
                            if (P.accumulate || where.half) tma_reduce_add_2d(&map_out, stage, (int32_t)c, wrow);
                            else tma_store_2d(&map_out, stage, (int32_t)c, wrow);
                            bulk_commit();
                        }
                    } else {
                        __syncwarp();
                        const int32_t rows = (int32_t)min((int64_t)32, P.M - wrow);
                        if (P.out_bf16) {
                            __nv_bfloat16* dst = (__nv_bfloat16*)P.out + (int64_t)wrow * P.ldo + c + lane;
                            if (c + lane < P.N) {
#pragma unroll 4
                                for (int32_t r = 0; r < rows; ++r, dst += P.ldo)
                                    *dst = *reinterpret_cast<const __nv_bfloat16*>(staged + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + 2 * (lane & 7));
                            }
                        } else {
                            const int col = lane & 15;
                            float* dst = (float*)P.out + (int64_t)(wrow + (lane >> 4)) * P.ldo + c + col;
                            if (c + col < P.N) {
#pragma unroll 4
                                for (int32_t r = lane >> 4; r < rows; r += 2, dst += 2 * P.ldo) {
                                    const float f = *reinterpret_cast<const float*>(staged + r * 64 + (((col >> 2) ^ ((r >> 1) & 3)) << 4) + 4 * (col & 3));
                                    *dst = P.accumulate ? __fadd_rn(*dst, f) : f;
                                }
                            }
                        }
                    }
                }
            }
        }
    }

    if (warp >= 4 && lane == 0) bulk_wait_all();
    __syncwarp();
    tc_fence_before();
    cluster_sync();                      // nobody leaves while the other CTA may still address this one
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<2>(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------
// few tokens: weights as the M side, tokens as the N side, the contraction cut over a cluster
// ------------------------------------------------------------------------------------------
template <int BN, bool GLU>
struct SmallCfg {
    static constexpr int W_BYTES = 128 * GB_K;                             // one weight tile
    static constexpr int STAGE_BYTES = W_BYTES * (GLU ? 2 : 1) + BN * GB_K;
    static constexpr int FIT = (int)(200 * 1024 / STAGE_BYTES);
    static constexpr int STAGES = FIT > 12 ? 12 : FIT;
    static constexpr int COLS = BN * (GLU ? 2 : 1);                         // TMEM columns of one k-block's sums
    static constexpr int BUFS = 512 / COLS > 4 ? 4 : 512 / COLS;
    static constexpr int TMEM = BUFS * COLS < 32 ? 32 : BUFS * COLS;
    static_assert((size_t)STAGES * STAGE_BYTES >= (size_t)COLS * 128 * 4, "the ring holds the partial sums afterwards");
    // Warps that add up: four, or eight that share the columns (the gated block: one half the gate, the other the up
    // projection).  With four a k-block of 128 tokens took 0.83 us, with eight 0.62.
    static constexpr int GROUPS = COLS >= 64 ? 2 : 1;
    static constexpr int EW = 4 * GROUPS, THREADS = 64 + 32 * EW;
    static constexpr int MY_COLS = COLS / GROUPS;                           // sums per thread
    static constexpr int MY_TOKENS = GLU ? BN : BN / GROUPS;                // tokens whose step sizes a warp needs
};
template <int BN, bool GLU>
struct SmallTail {
    using C = SmallCfg<BN, GLU>;
    uint64_t full[C::STAGES], empty[C::STAGES], tmem_full[C::BUFS], tmem_empty[C::BUFS], drain;
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    alignas(16) float token_scale[C::EW][4][C::MY_TOKENS];           // [warp][k-block of the chunk][token]
};
template <int BN, bool GLU>
constexpr size_t small_smem() { return 1024 + (size_t)SmallCfg<BN, GLU>::STAGES * SmallCfg<BN, GLU>::STAGE_BYTES + sizeof(SmallTail<BN, GLU>); }

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 f;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(addr) : "memory");
    return f;
}
__device__ __forceinline__ uint32_t cluster_nctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

// a: tokens [M], b (and b2): weights [N].  Cluster of S CTAs along x: CTA r takes k-blocks [r per, (r + 1) per).
template <int BN, bool GLU>
__global__ void __launch_bounds__(SmallCfg<BN, GLU>::THREADS, 1)
gemm_blocks_small_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                         const __grid_constant__ CUtensorMap map_b2, const __grid_constant__ GemmBlocksParams P) {
    pdl_trigger();                       // the wait follows the set-up below, which touches only shared memory and TMEM
    using C = SmallCfg<BN, GLU>;
    constexpr int STAGES = C::STAGES, BUFS = C::BUFS;
    using Tail = SmallTail<BN, GLU>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Tail* T = (Tail*)(smem + (size_t)STAGES * C::STAGE_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&T->full[s], 1); mbar_init(&T->empty[s], 1); }
        for (int b = 0; b < BUFS; ++b) { mbar_init(&T->tmem_full[b], 1); mbar_init(&T->tmem_empty[b], C::EW); }
        mbar_init(&T->drain, 1);
        T->abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<1>(&T->tmem_base, C::TMEM);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = T->tmem_base;
    const uint32_t rank = cluster_ctarank(), parts = cluster_nctarank();
    pdl_wait();

    const int32_t tn = (int32_t)(blockIdx.x / parts);                      // weight tile
    const int64_t n0 = (int64_t)tn * 128, t0 = (int64_t)blockIdx.y * BN;   // first weight row, first token
    const int32_t per = (P.num_kb + (int32_t)parts - 1) / (int32_t)parts;
    const int32_t kb0 = (int32_t)rank * per, kb1 = min(kb0 + per, P.num_kb);

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int32_t kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
                if (!mbar_wait(&T->empty[s], ph ^ 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                mbar_expect_tx(&T->full[s], C::STAGE_BYTES);
                const uint32_t bar = smem_u32(&T->full[s]);
                uint8_t* st = smem + (size_t)s * C::STAGE_BYTES;
                tma_load_2d<1>(st, &map_b, kb * GB_K, (int32_t)n0, bar);
                if constexpr (GLU) tma_load_2d<1>(st + C::W_BYTES, &map_b2, kb * GB_K, (int32_t)n0, bar);
                tma_load_2d<1>(st + C::W_BYTES * (GLU ? 2 : 1), &map_a, kb * GB_K, (int32_t)t0, bar);
            }
            if (!ok) {
                const uint32_t back = it < (uint32_t)STAGES ? it : (uint32_t)STAGES;
                for (uint32_t j = 1; j <= back; ++j) {
                    const uint32_t jt = it - j;
                    const uint64_t w0 = global_ns();
                    while (!mbar_try_wait(&T->full[jt % STAGES], (jt / STAGES) & 1u) && global_ns() - w0 < WAIT_LIMIT_NS) {}
                }
            }
        }
    } else if (warp == 1) {
        // the whole warp walks the loop, one elected lane issues (see the pair kernel)
        constexpr uint32_t idesc = make_idesc(1, 128, BN);
        const uint32_t elected = elect_one();
        uint32_t s = 0, ph = 0, buf = 0, buf_ph = 1;
        const uint64_t desc0 = make_smem_desc(smem_u32(smem));
        bool ok = true;
        for (int32_t kb = kb0; kb < kb1; ++kb) {
            ok = mbar_wait(&T->full[s], ph, &T->abort_flag) && mbar_wait(&T->tmem_empty[buf], buf_ph, &T->abort_flag);
            ok = !__any_sync(0xFFFFFFFFu, !ok);
            if (!ok) { gb_give_up(&T->abort_flag, P.status); break; }
            tc_fence_after();
            const uint64_t dw = desc0 + (uint64_t)(s * (C::STAGE_BYTES >> 4)), dx = dw + (uint64_t)((C::W_BYTES * (GLU ? 2 : 1)) >> 4);
            const uint32_t d = tmem_base + buf * C::COLS;
            if (elected) {
#pragma unroll
                for (int k = 0; k < GB_K / GB_UMMA_K; ++k) {
                    const uint64_t o = (uint64_t)((k * GB_UMMA_K) >> 4);
                    umma<1, 1>(d, dw + o, dx + o, idesc, k ? 1u : 0u);
                    if constexpr (GLU) umma<1, 1>(d + BN, dw + (uint64_t)(C::W_BYTES >> 4) + o, dx + o, idesc, k ? 1u : 0u);
                }
                umma_commit<1>(&T->tmem_full[buf], false);
                umma_commit<1>(&T->empty[s], false);
            }
            __syncwarp();
            s = s + 1 == (uint32_t)STAGES ? 0u : s + 1;
            ph ^= s == 0u ? 1u : 0u;
            buf = buf + 1 == (uint32_t)BUFS ? 0u : buf + 1;
            buf_ph ^= buf == 0u ? 1u : 0u;
        }
        if (!ok && elected) {
            umma_commit<1>(&T->drain, false);
            const uint64_t w0 = global_ns();
            while (!mbar_try_wait(&T->drain, 0u) && global_ns() - w0 < WAIT_LIMIT_NS) {}
        }
    } else {
        const int quarter = warp & 3, ew = warp - 2, grp = ew >> 2;
        const int wrow = quarter * 32 + lane;              // weight row within the tile = TMEM lane
        const int64_t n = n0 + wrow;
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + grp * C::MY_COLS;
        // one projection per thread, or both (gate columns, then up columns)
        constexpr bool BOTH = GLU && C::GROUPS == 1;
        const Blocks& wb = GLU && C::GROUPS == 2 && grp == 1 ? P.b2 : P.b;
        const int64_t wr = wb.tile_rows > 1 ? tn : n;
        const float* rw = n < P.N ? wb.scale + wr * wb.ld_scale : nullptr;
        const float* rw2 = BOTH && n < P.N ? P.b2.scale + wr * P.b2.ld_scale : nullptr;
        const int tok0 = GLU ? 0 : grp * C::MY_TOKENS;     // first of this warp's tokens
        constexpr int TPL = (C::MY_TOKENS + 31) / 32;      // tokens whose step sizes this lane fetches
        const float* rt[TPL];
#pragma unroll
        for (int i = 0; i < TPL; ++i) {
            const int64_t t = t0 + tok0 + lane + 32 * i;
            rt[i] = (lane + 32 * i < C::MY_TOKENS && t < P.M) ? P.a.scale + (P.a.tile_rows > 1 ? t / QBLK : t) * P.a.ld_scale : nullptr;
        }
        float (*ts)[C::MY_TOKENS] = T->token_scale[ew];
        float2 acc[C::MY_COLS / 2];
#pragma unroll
        for (int i = 0; i < C::MY_COLS / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
        float4 nw = scales4(rw, kb0 >> 2, P.num_kb, P.b_vec), nw2 = scales4(rw2, kb0 >> 2, P.num_kb, P.b_vec);
        float4 nt[TPL];
#pragma unroll
        for (int i = 0; i < TPL; ++i) nt[i] = scales4(rt[i], kb0 >> 2, P.num_kb, P.a_vec);
        float4 cw = nw, cw2 = nw2;
        uint32_t buf = 0, buf_ph = 0;
#pragma unroll 1
        for (int32_t kb = kb0; kb < kb1; ++kb) {
            const int32_t in4 = kb & 3;
            if (in4 == 0 || kb == kb0) {
                cw = nw; cw2 = nw2;
                __syncwarp();                              // the previous chunk has been read
#pragma unroll
                for (int i = 0; i < TPL; ++i) {
                    const int t = lane + 32 * i;
                    if (t < C::MY_TOKENS) { ts[0][t] = nt[i].x; ts[1][t] = nt[i].y; ts[2][t] = nt[i].z; ts[3][t] = nt[i].w; }
                }
                __syncwarp();
                const int32_t next = (kb >> 2) + 1;
                nw = scales4(rw, next, P.num_kb, P.b_vec);
                if constexpr (BOTH) nw2 = scales4(rw2, next, P.num_kb, P.b_vec);
#pragma unroll
                for (int i = 0; i < TPL; ++i) nt[i] = scales4(rt[i], next, P.num_kb, P.a_vec);
            }
            const float sw = pick4(cw, in4), sw2 = pick4(cw2, in4);
            wait_or_abort(smem_u32(&T->tmem_full[0]) + 8 * buf, buf_ph, &T->abort_flag, P.status);
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < C::MY_COLS / 16; ++c) {
                uint32_t v[16];
                tmem_ld16(taddr + buf * C::COLS + 16 * c, v);
                tmem_ld_wait();
                const float s = BOTH && c >= BN / 16 ? sw2 : sw;
                const float2 s2 = make_float2(s, s);
                const float* tk = &ts[in4][(16 * c) % C::MY_TOKENS];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 f = *reinterpret_cast<const float4*>(tk + 4 * q);
                    float2& x = acc[8 * c + 2 * q];
                    float2& y = acc[8 * c + 2 * q + 1];
                    x = __ffma2_rn(pair(v[4 * q], v[4 * q + 1]), __fmul2_rn(make_float2(f.x, f.y), s2), x);
                    y = __ffma2_rn(pair(v[4 * q + 2], v[4 * q + 3]), __fmul2_rn(make_float2(f.z, f.w), s2), y);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&T->tmem_empty[buf]);
            buf = buf + 1 == (uint32_t)BUFS ? 0u : buf + 1;
            buf_ph ^= buf == 0u ? 1u : 0u;
        }
        // this CTA's part of every sum: [token (gate, then up)][weight row], in the ring, which nothing uses any more
        float* part = reinterpret_cast<float*>(smem) + grp * C::MY_COLS * 128;
#pragma unroll
        for (int i = 0; i < C::MY_COLS / 2; ++i) { part[2 * i * 128 + wrow] = acc[i].x; part[(2 * i + 1) * 128 + wrow] = acc[i].y; }
    }

    __syncwarp();
    tc_fence_before();
    cluster_sync();                      // all parts are there
    if (warp >= 2) {
        // token t of the tile belongs to CTA t % parts and to one of its warps; a lane takes four columns.  A warp works on
        // several tokens at a time: each is a chain of dependent steps (loads, maxima, quotients) of over a thousand cycles.
        // (With sixteen tokens at most there is little to overlap, and the longer code costs more: 8.4 us became 10.1.)
        constexpr int U = BN == 16 ? 1 : GLU ? 4 : 2;
        const int64_t c = n0 + 4 * lane;
        const uint32_t base = smem_u32(smem) + (uint32_t)lane * 16u;
        const int64_t tokens = P.M - t0 < BN ? P.M - t0 : BN;
        const int stride = (int)parts * C::EW;
        for (int t = (int)rank + (int)parts * (warp - 2); t < tokens; t += U * stride) {
            float x[U][4], y[U][4];
            auto gather = [&](float (&sum)[4], uint32_t addr) {            // all parts' loads are in flight before the first addition
                float4 f[8];
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (i < parts) f[i] = ld_cluster_f4(map_to_cta(addr, i));
                sum[0] = sum[1] = sum[2] = sum[3] = 0.0f;
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (i < parts) { sum[0] += f[i].x; sum[1] += f[i].y; sum[2] += f[i].z; sum[3] += f[i].w; }
            };
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int ti = t + i * stride < tokens ? t + i * stride : t;       // past the end: a token done already, not stored
                gather(x[i], base + (uint32_t)ti * 512u);
                if constexpr (GLU) gather(y[i], base + (uint32_t)(BN + ti) * 512u);
            }
            if constexpr (GLU) {
                auto emit = [&](const Blocks& o, const float (&val)[U][4]) {
                    if (!o.codes) return;
                    uint32_t m[U];
#pragma unroll
                    for (int i = 0; i < U; ++i)
                        m[i] = __reduce_max_sync(0xFFFFFFFFu, abs_word(absmax3(absmax3(val[i][0], val[i][1], val[i][2]), val[i][3], 0.0f)));
                    // lane i has the divisions of token i
                    uint32_t mine = m[0];
#pragma unroll
                    for (int i = 1; i < U; ++i) mine = lane == i ? m[i] : mine;
                    const float inv = block_inv(mine);
                    const int t_mine = t + lane * stride;
                    if (lane < U && t_mine < tokens) {
                        o.scale[(t0 + t_mine) * o.ld_scale + tn] = block_size(mine);
                        if (block_nonfinite(mine)) note(P.status, SRQ_ERR_NONFINITE);
                    }
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        const float f = __shfl_sync(0xFFFFFFFFu, inv, i);
                        const uint32_t w = encode4<false>(val[i][0], val[i][1], val[i][2], val[i][3], f, f, f, f, 0, 0, 0, 0);
                        if (t + i * stride >= tokens) continue;
                        uint8_t* dst = o.codes + (t0 + t + i * stride) * o.ld + c;
                        if (c + 4 <= P.N) *reinterpret_cast<uint32_t*>(dst) = w;
                        else
                            for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = (uint8_t)(w >> (8 * e));
                    }
                };
                emit(P.gate, x);
                emit(P.up, y);
#pragma unroll
                for (int i = 0; i < U; ++i) {
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float2 g2 = make_float2(x[i][e], x[i][e + 1]), u2 = make_float2(y[i][e], y[i][e + 1]);
                        const float2 h2 = P.gelu ? gated2<true>(g2, u2) : gated2<false>(g2, u2);
                        x[i][e] = h2.x; x[i][e + 1] = h2.y;
                    }
                }
                emit(P.h, x);
            }
            if (P.out) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int64_t row = t0 + t + i * stride;
                    if (t + i * stride >= tokens) continue;
                    float (&v)[4] = x[i];
                    if (P.out_bf16) {
                        __nv_bfloat16* dst = (__nv_bfloat16*)P.out + row * P.ldo + c;
                        if (P.h_vec && c + 4 <= P.N) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                        else
                            for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = __float2bfloat16_rn(v[e]);
                    } else {
                        float* dst = (float*)P.out + row * P.ldo + c;
                        if (P.accumulate)
                            for (int e = 0; e < 4; ++e) if (c + e < P.N) v[e] = __fadd_rn(dst[e], v[e]);
                        if (P.h_vec && c + 4 <= P.N) *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
                        else
                            for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = v[e];
                    }
                }
            }
        }
    }
    cluster_sync();                      // nobody leaves while its parts are still being read
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<1>(tmem_base, C::TMEM);
    }
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static bool encode_codes(CUtensorMap* map, const Blocks& b, int64_t rows, int64_t cols, int box_rows) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)b.ld};
    cuuint32_t box[2] = {(cuuint32_t)GB_K, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)b.codes, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// What leaves through block stores: boxes of 32 rows, 64 bytes of binary32 or bfloat16 (esize 4 or 2) or 32 codes (esize 1) wide.
static bool encode_result(CUtensorMap* map, void* base, unsigned esize, int64_t rows, int64_t cols, int64_t ld) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * esize};
    cuuint32_t box[2] = {esize == 1 ? 32u : 64u / esize, 32};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, esize == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : esize == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
               base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, esize == 1 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_64B,
               CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Per device: SM count, resident CTA pairs, resident clusters of the few-token kernel by cluster size.
struct BlocksDevice { bool ready = false; int sms = 1, pairs = 0, clusters[9] = {}; };

template <typename K>
static bool opt_in(K kernel, size_t smem) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess;
}
template <int BN>
static bool opt_in_small() {
    if (!opt_in(gemm_blocks_small_kernel<BN, false>, small_smem<BN, false>())) return false;
    if constexpr (BN <= 64) return opt_in(gemm_blocks_small_kernel<BN, true>, small_smem<BN, true>());
    return true;
}

static bool blocks_device(BlocksDevice** out) {
    static BlocksDevice info[64];
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    std::lock_guard<std::mutex> lock(mu);
    BlocksDevice& d = info[dev];
    if (!d.ready) {
        if (cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || d.sms <= 0) return false;
        if (!opt_in(gemm_blocks_kernel<false, false>, gb_smem()) || !opt_in(gemm_blocks_kernel<false, true>, gb_smem()) ||
            !opt_in(gemm_blocks_kernel<true, false>, gb_smem()) || !opt_in(gemm_blocks_kernel<true, true>, gb_smem()) ||
            !opt_in_small<16>() || !opt_in_small<32>() || !opt_in_small<64>() || !opt_in_small<128>())
            return false;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
        cfg.attrs = &at; cfg.numAttrs = 1;
        int n = 0;
        at.val.clusterDim.x = 2;
        cfg.gridDim = dim3((unsigned)(d.sms / 2 * 2)); cfg.blockDim = dim3(GB_THREADS); cfg.dynamicSmemBytes = gb_smem();
        if (cudaOccupancyMaxActiveClusters(&n, gemm_blocks_kernel<false, false>, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
        d.pairs = n < d.sms / 2 ? n : d.sms / 2;
        for (int s = 1; s <= 8; ++s) {
            at.val.clusterDim.x = (unsigned)s;
            cfg.gridDim = dim3((unsigned)(d.sms / s * s)); cfg.blockDim = dim3(SmallCfg<16, false>::THREADS); cfg.dynamicSmemBytes = small_smem<16, false>();
            if (cudaOccupancyMaxActiveClusters(&n, gemm_blocks_small_kernel<16, false>, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
            d.clusters[s] = n;
        }
        d.ready = true;
    }
    *out = &d;
    return true;
}

// Which kernel, and how its tiles are cut.  Both kernels' time is modelled in units of 10 ns from measurements (N and K of 512
// to 4096; the products of a whole family of sizes are within a fifth of it):
//   few tokens   rounds (k-blocks of a part x cost(bn) + 300 + cost(part) (parts - 1)), where a k-block costs a CTA 28 / 38 /
//                42 / 62 with tiles of 16 / 32 / 64 / 128 tokens (gated: 45 / 48 / 67, and 4 per token of its share for
//                the epilogue), a further part of the contraction 20 (gated: 50) for the exchange, and a round is what is
//                resident at a time
//   CTA pairs    rounds x k-blocks x 55 + 400 (gated: + 250 per round for its longer epilogue)
// 333 tokens, 2048 -> 2560: pairs 13.7 us on 20 of 74 pairs, tiles of 64 tokens 11.0; 1024 tokens, 512 outputs: 12.9 and 7.8;
// 1024 tokens, 2048 -> 2560: 14.3 and 35; gated, 64 tokens, 2048 -> 5632: 16.3 and 13.3, 128 tokens: 16.8 and 20.6.
// halve: the result may be added up from two parts (binary32, overwritten, stored in blocks): tiles of a last round that fills
// at most half of the pairs are done in two halves of the contraction, at the cost of clearing their rows before.
// 5632 x 2048 x 8192, 176 tiles on 74 pairs: two and a half rounds instead of three.
struct Plan { bool pairs; int bn, parts; bool halves; };
static Plan plan_product(const BlocksDevice& d, int64_t M, int64_t N, int32_t num_kb, bool glu, bool halve) {
    Plan best = {true, 0, 0, false};
    const int64_t cols = glu ? 128 : GB_N, tiles = ((M + 2 * GB_M - 1) / (2 * GB_M)) * ((N + cols - 1) / cols);
    const int64_t per_round = (int64_t)num_kb * 55 + (glu ? 250 : 0);
    int64_t cost = d.pairs > 0 ? (tiles + d.pairs - 1) / d.pairs * per_round + 400 : INT64_MAX;
    if (halve && d.pairs > 0 && num_kb >= 16 && tiles % d.pairs != 0 && 2 * (tiles % d.pairs) <= d.pairs) {
        const int64_t c = tiles / d.pairs * per_round + per_round / 2 + 700;
        if (c < cost) { cost = c; best.halves = true; }
    }
    static const int kCost[2][4] = {{28, 38, 42, 62}, {45, 48, 67, 0}};
    for (int i = 0; i < (glu ? 3 : 4); ++i) {
        const int bn = 16 << i;
        if (i > 0 && bn / 2 >= M) break;                             // half as many would do
        const int64_t n = ((N + 127) / 128) * ((M + bn - 1) / bn);
        if ((M + bn - 1) / bn > 65535) continue;                     // grid limit
        for (int s = 1; s <= 8 && s <= num_kb; ++s) {
            if (d.clusters[s] <= 0) continue;
            const int32_t per = (num_kb + s - 1) / s;
            if ((num_kb + per - 1) / per != s) continue;             // a part would be empty
            const int64_t c = (n + d.clusters[s] - 1) / d.clusters[s] * ((int64_t)per * kCost[glu][i] + 300 + (glu ? 50 : 20) * (s - 1) + (glu ? 4 * (M < bn ? M : bn) / s : 0));
            if (c < cost) { cost = c; best = {false, bn, s, false}; }
        }
    }
    return best;
}

static bool scale_vec(const Blocks& b) { return (uintptr_t)b.scale % 16 == 0 && b.ld_scale % 4 == 0; }

template <int BN, bool GLU>
static cudaError_t launch_small_bn(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mb2, const GemmBlocksParams& P,
                                   int parts, int64_t tiles_n, int64_t tiles_t, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles_n * parts), (unsigned)tiles_t); cfg.blockDim = dim3(SmallCfg<BN, GLU>::THREADS);
    cfg.dynamicSmemBytes = small_smem<BN, GLU>(); cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = (unsigned)parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = pdl_allowed(stream) ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_blocks_small_kernel<BN, GLU>, ma, mb, mb2, P);
}

template <bool GLU, bool COLV>
static cudaError_t launch_pair(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mb2, const CUtensorMap& mo,
                               const CUtensorMap& mg, const CUtensorMap& mu, const GemmBlocksParams& P, unsigned pairs, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pairs * 2); cfg.blockDim = dim3(GB_THREADS); cfg.dynamicSmemBytes = gb_smem(); cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = pdl_allowed(stream) ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_blocks_kernel<GLU, COLV>, ma, mb, mb2, mo, mg, mu, P);
}

static srq_status_t run_small(const Plan& plan, GemmBlocksParams& P, bool glu, int64_t Kc, cudaStream_t stream) {
    const int bn = plan.bn, parts = plan.parts;
    const int64_t tiles_n = (P.N + 127) / 128, tiles_t = (P.M + bn - 1) / bn;
    CUtensorMap ma, mb, mb2;
    if (!encode_codes(&ma, P.a, P.M, Kc, bn) || !encode_codes(&mb, P.b, P.N, Kc, 128)) return SRQ_ERR_CUDA;
    mb2 = mb;
    if (glu && !encode_codes(&mb2, P.b2, P.N, Kc, 128)) return SRQ_ERR_CUDA;
    const int esize = P.out_bf16 ? 2 : 4;
    P.h_vec = P.out && (uintptr_t)P.out % (4 * esize) == 0 && P.ldo % 4 == 0;       // four results per lane
    cudaError_t e;
    if (glu) {
        e = bn == 16 ? launch_small_bn<16, true>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream)
          : bn == 32 ? launch_small_bn<32, true>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream)
                     : launch_small_bn<64, true>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream);
    } else {
        e = bn == 16 ? launch_small_bn<16, false>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream)
          : bn == 32 ? launch_small_bn<32, false>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream)
          : bn == 64 ? launch_small_bn<64, false>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream)
                     : launch_small_bn<128, false>(ma, mb, mb2, P, parts, tiles_n, tiles_t, stream);
    }
    count_launch();
    return e == cudaSuccess ? SRQ_OK : SRQ_ERR_CUDA;
}

// The result leaves through block stores: 16-byte aligned rows that also end on a 16-byte boundary (a block store that reaches
// over the map's edge may write the whole last 16-byte piece).
static bool block_stores(const GemmBlocksParams& P) {
    const int per16 = P.out_bf16 ? 8 : 4;
    return P.out && (uintptr_t)P.out % 16 == 0 && P.ldo % per16 == 0 && P.N % per16 == 0;
}

static srq_status_t run_pairs(const BlocksDevice& d, const Plan& plan, GemmBlocksParams& P, bool glu, int64_t Kc, cudaStream_t stream) {
    if (d.pairs <= 0) return SRQ_ERR_UNSUPPORTED;
    P.tiles_m = (int32_t)((P.M + 2 * GB_M - 1) / (2 * GB_M));
    P.tiles_n = (int32_t)((P.N + (glu ? 128 : GB_N) - 1) / (glu ? 128 : GB_N));
    CUtensorMap ma, mb, mb2, mo, mg, mu;
    if (!encode_codes(&ma, P.a, P.M, Kc, GB_M) || !encode_codes(&mb, P.b, P.N, Kc, 64)) return SRQ_ERR_CUDA;
    mb2 = mb; mo = mb; mg = mb; mu = mb;
    if (glu && !encode_codes(&mb2, P.b2, P.N, Kc, 64)) return SRQ_ERR_CUDA;
    P.h_vec = P.out && (uintptr_t)P.out % 16 == 0 && P.ldo % (P.out_bf16 ? 8 : 4) == 0;
    if (!glu) P.tma_out = block_stores(P) && encode_result(&mo, P.out, P.out_bf16 ? 2 : 4, P.M, P.N, P.ldo);
    else
        P.tma_out = P.N % 16 == 0 && (!P.h.codes || encode_result(&mo, P.h.codes, 1, P.M, P.N, P.h.ld)) &&
                    (!P.gate.codes || encode_result(&mg, P.gate.codes, 1, P.M, P.N, P.gate.ld)) &&
                    (!P.up.codes || encode_result(&mu, P.up.codes, 1, P.M, P.N, P.up.ld));
    const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n;
    if (2 * tiles > INT32_MAX) return SRQ_ERR_UNSUPPORTED;
    P.full_tiles = (int32_t)tiles;
    if (plan.halves && P.tma_out) {
        P.full_tiles = (int32_t)(tiles / d.pairs * d.pairs);
        P.half_kb = (P.num_kb / 2 + 3) / 4 * 4;                  // step sizes come in chunks of four
        const int64_t first = (int64_t)(P.full_tiles / P.tiles_n) * 2 * GB_M;      // whole tiles in these rows are overwritten
        if (cudaMemset2DAsync((float*)P.out + first * P.ldo, (size_t)P.ldo * 4, 0, (size_t)P.N * 4, (size_t)(P.M - first), stream) != cudaSuccess)
            return SRQ_ERR_CUDA;
    }
    const int64_t units = P.full_tiles + 2 * (tiles - P.full_tiles);
    const unsigned pairs = (unsigned)(units < d.pairs ? units : d.pairs);
    const bool colv = P.b.tile_rows == 1;
    cudaError_t e;
    if (glu) e = colv ? launch_pair<true, true>(ma, mb, mb2, mo, mg, mu, P, pairs, stream) : launch_pair<true, false>(ma, mb, mb2, mo, mg, mu, P, pairs, stream);
    else e = colv ? launch_pair<false, true>(ma, mb, mb2, mo, mg, mu, P, pairs, stream) : launch_pair<false, false>(ma, mb, mb2, mo, mg, mu, P, pairs, stream);
    count_launch();
    return e == cudaSuccess ? SRQ_OK : SRQ_ERR_CUDA;
}

static srq_status_t run_product(const BlocksDevice& d, GemmBlocksParams& P, bool glu, int64_t Kc, cudaStream_t stream) {
    const bool halve = !glu && !P.out_bf16 && !P.accumulate && block_stores(P);
    const Plan plan = plan_product(d, P.M, P.N, P.num_kb, glu, halve);
    return plan.pairs ? run_pairs(d, plan, P, glu, Kc, stream) : run_small(plan, P, glu, Kc, stream);
}

srq_status_t launch_gemm_blocks(const GemmBlocksArgs& g, uint32_t* status, cudaStream_t stream) {
    BlocksDevice* d = nullptr;
    if (!blocks_device(&d)) return SRQ_ERR_CUDA;
    GemmBlocksParams P = {};
    P.M = g.M; P.N = g.N; P.num_kb = (int32_t)((g.Kc + GB_K - 1) / GB_K);
    P.a = g.a; P.b = g.b; P.a_vec = scale_vec(g.a); P.b_vec = scale_vec(g.b);
    P.out = g.out; P.ldo = g.ldo; P.out_bf16 = g.out_dt == SRQ_BF16; P.accumulate = g.accumulate;
    P.status = status;
    return run_product(*d, P, false, g.Kc, stream);
}

srq_status_t launch_glu_fwd(const GluArgs& g, uint32_t* status, cudaStream_t stream) {
    BlocksDevice* d = nullptr;
    if (!blocks_device(&d)) return SRQ_ERR_CUDA;
    GemmBlocksParams P = {};
    P.M = g.T; P.N = g.F; P.num_kb = (int32_t)((g.K + GB_K - 1) / GB_K);
    P.a = g.x; P.b = g.wg; P.b2 = g.wu; P.a_vec = scale_vec(g.x); P.b_vec = scale_vec(g.wg) && scale_vec(g.wu);
    P.out = g.h_out; P.ldo = g.ld_h; P.out_bf16 = g.h_dt == SRQ_BF16;
    P.h = g.h; P.gate = g.gate; P.up = g.up; P.gelu = g.act == SRQ_GELU;
    P.status = status;
    return run_product(*d, P, true, g.K, stream);
}

}  // namespace srq
