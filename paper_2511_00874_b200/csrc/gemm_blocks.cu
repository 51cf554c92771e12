// Products of block-coded E4M3 matrices on the 5th-generation tensor cores, and the gated feed-forward block
// as an epilogue of the same kernels.
//
//   out[i, j] = sum_k sA[i, k] sB[j, k] P_k[i, j],     P_k = the 128-long piece k of the contraction
//
// The step sizes change every 128 values of the contraction, so the tensor core cannot add up the whole sum:
// each P_k is left in TMEM for itself (kind::f8f6f4, binary32), read back and added into binary32 registers
// with its factor.  That takes one tcgen05.ld and one multiply-add per element and k-block, next to the 512
// cycles the MMAs of a 128 x 256 x 128 piece take: the two run side by side, k-block by k-block, through
// two TMEM buffers.
//
// gemm_blocks_kernel: 256 x 256 tiles on CTA pairs (tcgen05.mma.cta_group::2, M256 N256 K32), persistent.
//   warp 0      TMA producer (128-byte swizzled tiles, ring of 5 stages of 32 KB)
//   warp 1      TMEM and MMA issue (leader CTA): one k-block into one TMEM buffer at a time, in turn
//   warps 4-11  two groups of four; a thread owns one row of the CTA's 128 and 128 of the 256 columns: group
//               g columns 128 g .. in a plain product; in the gated block, whose 256 columns are 128 of the
//               gate and 128 of the up projection (one CTA of the pair stages Wg, the other Wu), columns
//               64 g .. 64 g + 63 of both, so that g and u of an element meet in one thread
// gemm_blocks_small_kernel: few tokens.  The roles turn around: 128 rows of the weights are the M of the MMA and
// 16 to 128 tokens its N, the contraction is cut over a cluster of CTAs (as many as fill the machine), and the
// parts are added through distributed shared memory in a fixed order.  Reading the weights once is all there
// is to do, and every SM reads its share with up to 200 KB in flight.
//
// Every wait is bounded (2 s); on expiry SRQ_ERR_TIMEOUT is recorded, all roles run to their end without
// waiting any more, and TMEM is freed.
#include <cuda.h>

#include <mutex>

#include "blocks.cuh"
#include "tensor_core.cuh"

namespace srq {

constexpr int GB_M = 128, GB_N = 256, GB_K = 128;      // rows per CTA, tile columns, bytes (= codes) per k-block
constexpr int GB_STAGES = 5;
constexpr int GB_STAGE_BYTES = GB_M * GB_K + (GB_N / 2) * GB_K;
constexpr int GB_THREADS = 384;
// Registers: 384 threads start with 168 each; the first warpgroup keeps 40 and the two that hold 128 sums per
// thread take 232 (40 + 2 x 232 = 3 x 168: exactly what the block was launched with).
constexpr int GB_REGS_FEW = 40, GB_REGS_MANY = 232;
constexpr int GB_OUT_BYTES = 32 * 128;                 // staging block of an epilogue warp
constexpr int GB_UMMA_K = 32;

struct GemmBlocksParams {
    int64_t M, N;                       // N: columns of out, or of h (the gated block's F)
    int32_t num_kb, tiles_m, tiles_n;
    Blocks a, b, b2;                    // b2: up projection of the gated block
    int32_t a_vec, b_vec;               // 16-byte loads of four step sizes allowed
    void* out; int64_t ldo; int32_t out_bf16, tma_out, accumulate;
    Blocks h, gate, up;                 // gated block
    int32_t gelu, h_vec;
    uint32_t* status;
};

struct GbTail {
    uint64_t full[GB_STAGES], empty[GB_STAGES], tmem_full[2], tmem_empty[2], drain;
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    alignas(16) float col_scale[2][2][4][128];     // [group][chunk parity][k-block of the chunk][column]
    uint32_t amax[2][3][2][GB_M];                  // gated block: [tile parity][which][group][row]
};
constexpr size_t gb_smem() { return 1024 + (size_t)GB_STAGES * GB_STAGE_BYTES + 8 * GB_OUT_BYTES + sizeof(GbTail); }

__device__ __forceinline__ void gb_give_up(volatile uint32_t* abort_flag, uint32_t* status) {
    *abort_flag = 1u;
    note(status, SRQ_ERR_TIMEOUT);
}

// 32 lanes x 32 columns of TMEM, in registers once tmem_ready has passed (which ties the registers to the wait).
__device__ __forceinline__ void tmem_ready(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
          "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
          "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
          "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
        :: "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ready(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
          "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
        :: "memory");
}

// Step sizes of k-blocks 4 c .. 4 c + 3 of one scale row (zeros past num_kb).
__device__ __forceinline__ float4 scales4(const float* row, int32_t c, int32_t num_kb, bool vec) {
    const int32_t k = 4 * c;
    if (row == nullptr || k >= num_kb) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (vec && k + 4 <= num_kb) return __ldg(reinterpret_cast<const float4*>(row + k));
    float4 f = make_float4(__ldg(row + k), 0.0f, 0.0f, 0.0f);
    if (k + 1 < num_kb) f.y = __ldg(row + k + 1);
    if (k + 2 < num_kb) f.z = __ldg(row + k + 2);
    if (k + 3 < num_kb) f.w = __ldg(row + k + 3);
    return f;
}
__device__ __forceinline__ float pick4(const float4& f, int32_t i) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; }

// Sixty-four consecutive codes of a row from column c (rows start on 16-byte boundaries).
__device__ __forceinline__ void store_codes64(uint8_t* row, int64_t c, int64_t cols, const uint32_t (&w)[16]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (c + 16 * q + 16 <= cols) {
            *reinterpret_cast<uint4*>(row + c + 16 * q) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c + 16 * q + e < cols) row[c + 16 * q + e] = (uint8_t)(w[4 * q + (e >> 2)] >> (8 * (e & 3)));
        }
    }
}

// GLU: the gated block's epilogue instead of the plain one.  COLV: b has a step size per row (per column of
// out), not per 128 of them.
template <bool GLU, bool COLV>
__global__ void __launch_bounds__(GB_THREADS, 1)
gemm_blocks_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_b2, const __grid_constant__ CUtensorMap map_out,
                   const __grid_constant__ GemmBlocksParams P) {
    pdl_trigger();                       // the wait follows the set-up below, which touches only shared memory and TMEM
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* out_stage = smem + (size_t)GB_STAGES * GB_STAGE_BYTES;
    GbTail* T = (GbTail*)(out_stage + 8 * GB_OUT_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < GB_STAGES; ++s) { mbar_init(&T->full[s], 1); mbar_init(&T->empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&T->tmem_full[b], 1); mbar_init(&T->tmem_empty[b], 16); }   // 8 warps x 2 CTAs
        mbar_init(&T->drain, 1);
        T->abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<2>(&T->tmem_base, 512);
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = T->tmem_base;
    pdl_wait();

    const int64_t groups = gridDim.x / 2, group = blockIdx.x / 2;
    const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n;
    constexpr int TILE_COLS = GLU ? 128 : GB_N;        // columns of the result a tile covers

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
            for (int64_t u = group; u < tiles && ok; u += groups) {
                const int32_t tn = (int32_t)(u % P.tiles_n), tm = (int32_t)(u / P.tiles_n);
                const int32_t row_a = (tm * 2 + (int32_t)rank) * GB_M;
                const int32_t row_b = GLU ? tn * 128 : tn * GB_N + (int32_t)rank * 128;
                for (int32_t kb = 0; kb < P.num_kb; ++kb, ++it) {
                    const uint32_t s = it % GB_STAGES, ph = (it / GB_STAGES) & 1u;
                    if (!mbar_wait(&T->empty[s], ph ^ 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                    if (leader) mbar_expect_tx(&T->full[s], GB_STAGE_BYTES * 2);
                    const uint32_t bar = map_to_cta(smem_u32(&T->full[s]), 0);
                    uint8_t* sa = smem + (size_t)s * GB_STAGE_BYTES;
                    tma_load_2d<2>(sa, &map_a, kb * GB_K, row_a, bar);
                    tma_load_2d<2>(sa + GB_M * GB_K, mb, kb * GB_K, row_b, bar);
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
        if (lane == 0 && leader) {
            const uint32_t idesc = make_idesc(1, GB_M * 2, GB_N);
            bool ok = true, ready = false;
            uint32_t s = 0, ph = 0, it = 0;
            const uint64_t desc0 = make_smem_desc(smem_u32(smem));
            uint64_t da = desc0;
            for (int64_t u = group; u < tiles && ok; u += groups) {
                for (int32_t kb = 0; kb < P.num_kb; ++kb, ++it) {
                    const uint32_t buf = it & 1u, use = it >> 1;
                    if (!mbar_wait(&T->tmem_empty[buf], (use & 1u) ^ 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                    if (!ready && !mbar_wait(&T->full[s], ph, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                    tc_fence_after();
                    const uint32_t d_tmem = tmem_base + buf * GB_N;
                    const uint64_t db = da + (uint64_t)((GB_M * GB_K) >> 4);
                    const uint32_t ns = s + 1 == (uint32_t)GB_STAGES ? 0u : s + 1, nph = ns == 0u ? ph ^ 1u : ph;
                    umma<2, 1>(d_tmem, da, db, idesc, 0u);
                    ready = mbar_test_wait(&T->full[ns], nph);
#pragma unroll
                    for (int k = 1; k < GB_K / GB_UMMA_K; ++k)
                        umma<2, 1>(d_tmem, da + (uint64_t)((k * GB_UMMA_K) >> 4), db + (uint64_t)((k * GB_UMMA_K) >> 4), idesc, 1u);
                    umma_commit<2>(&T->empty[s], true);
                    umma_commit<2>(&T->tmem_full[buf], true);
                    s = ns; ph = nph;
                    da = ns == 0u ? desc0 : da + (uint64_t)(GB_STAGE_BYTES >> 4);
                }
            }
            if (!ok) {
                umma_commit<2>(&T->drain, false);
                const uint64_t t0 = global_ns();
                while (!mbar_try_wait(&T->drain, 0u) && global_ns() - t0 < WAIT_LIMIT_NS) {}
            }
        }
    }
    } else {
        // ------------------------------------------------------------------ scaling and epilogue (warps 4..11)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(GB_REGS_MANY));
        const int quarter = warp & 3, egrp = (warp - 4) >> 2, etid = (threadIdx.x - 128) & 127;
        const int trow = quarter * 32 + lane;            // row within this CTA's 128
        const uint32_t empty0 = map_to_cta(smem_u32(&T->tmem_empty[0]), 0), empty1 = map_to_cta(smem_u32(&T->tmem_empty[1]), 0);
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
        // first TMEM column of each 32-column piece this thread adds up
        auto piece = [&](int c) -> uint32_t { return GLU ? (uint32_t)((c >> 1) * 128 + 64 * egrp + 32 * (c & 1)) : (uint32_t)(128 * egrp + 32 * c); };
        const uint32_t stage = smem_u32(out_stage + (warp - 4) * GB_OUT_BYTES);
        bool ok = true;
        uint32_t it = 0, chunks = 0, par = 0;
        for (int64_t u = group; u < tiles; u += groups) {
            const int32_t tn = (int32_t)(u % P.tiles_n), tm = (int32_t)(u / P.tiles_n);
            const int64_t row0 = ((int64_t)tm * 2 + rank) * GB_M, row = row0 + trow;
            const int64_t col0 = (int64_t)tn * TILE_COLS;
            // this thread's scale rows
            const float* ra = row < P.M ? P.a.scale + (P.a.tile_rows > 1 ? row / QBLK : row) * P.a.ld_scale : nullptr;
            const float* rb = nullptr;                     // one step size per 128 columns ...
            const float* rb2 = nullptr;
            const float* rc = nullptr;                     // ... or this thread's share of the columns' own
            if constexpr (!COLV) {
                const int64_t tb = GLU ? tn : (int64_t)tn * 2 + egrp;
                if (tb * QBLK < P.N) {
                    rb = P.b.scale + tb * P.b.ld_scale;
                    if constexpr (GLU) rb2 = P.b2.scale + tb * P.b2.ld_scale;
                }
            } else {
                const int64_t c = GLU ? col0 + 64 * egrp + (etid & 63) : col0 + 128 * egrp + etid;
                const Blocks& w = GLU && etid >= 64 ? P.b2 : P.b;
                if (c < P.N) rc = w.scale + c * w.ld_scale;
            }
            float acc[128];
#pragma unroll
            for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
            float4 na = scales4(ra, 0, P.num_kb, P.a_vec), nb, nb2 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if constexpr (!COLV) {
                nb = scales4(rb, 0, P.num_kb, P.b_vec);
                if constexpr (GLU) nb2 = scales4(rb2, 0, P.num_kb, P.b_vec);
            } else {
                nb = scales4(rc, 0, P.num_kb, P.b_vec);
            }
            float4 ca = na, cb = nb, cb2 = nb2;
#pragma unroll 1
            for (int32_t kb = 0; kb < P.num_kb; ++kb, ++it) {
                const int32_t in4 = kb & 3, chunk = kb >> 2;
                if (in4 == 0) ++chunks;
                float (*cs)[128] = T->col_scale[egrp][chunks & 1];
                if (in4 == 0) {
                    ca = na; cb = nb; cb2 = nb2;
                    if constexpr (COLV) {
                        // the chunk before last is what this buffer held: every warp of the group has left it
                        cs[0][etid] = cb.x; cs[1][etid] = cb.y; cs[2][etid] = cb.z; cs[3][etid] = cb.w;
                        asm volatile("bar.sync %0, 128;" ::"r"(1 + egrp) : "memory");
                    }
                    na = scales4(ra, chunk + 1, P.num_kb, P.a_vec);
                    if constexpr (!COLV) {
                        nb = scales4(rb, chunk + 1, P.num_kb, P.b_vec);
                        if constexpr (GLU) nb2 = scales4(rb2, chunk + 1, P.num_kb, P.b_vec);
                    } else {
                        nb = scales4(rc, chunk + 1, P.num_kb, P.b_vec);
                    }
                }
                const float sa = pick4(ca, in4);
                float s0 = sa, s1 = sa;
                if constexpr (!COLV) {
                    s0 = __fmul_rn(sa, pick4(cb, in4));
                    if constexpr (GLU) s1 = __fmul_rn(sa, pick4(cb2, in4)); else s1 = s0;
                }
                const uint32_t buf = it & 1u, use = it >> 1;
                if (ok && !mbar_wait(&T->tmem_full[buf], use & 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; }
                if (__any_sync(0xFFFFFFFFu, !ok)) ok = false;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(taddr + buf * GB_N + piece(c), v);
                    tmem_ready(v);
                    if (c == 3) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(buf ? empty1 : empty0);
                    }
                    if constexpr (!COLV) {
                        const float s = c < 2 ? s0 : s1;
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[32 * c + i] = fmaf(__uint_as_float(v[i]), s, acc[32 * c + i]);
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const float4 f = *reinterpret_cast<const float4*>(&cs[in4][32 * c + 4 * q]);
                            acc[32 * c + 4 * q + 0] = fmaf(__uint_as_float(v[4 * q + 0]), sa * f.x, acc[32 * c + 4 * q + 0]);
                            acc[32 * c + 4 * q + 1] = fmaf(__uint_as_float(v[4 * q + 1]), sa * f.y, acc[32 * c + 4 * q + 1]);
                            acc[32 * c + 4 * q + 2] = fmaf(__uint_as_float(v[4 * q + 2]), sa * f.z, acc[32 * c + 4 * q + 2]);
                            acc[32 * c + 4 * q + 3] = fmaf(__uint_as_float(v[4 * q + 3]), sa * f.w, acc[32 * c + 4 * q + 3]);
                        }
                    }
                }
            }

            if constexpr (GLU) {
                // acc: 64 gate columns, then the same 64 up columns
                const int64_t f0 = col0 + 64 * egrp;
                const bool live = row < P.M;
                auto emit = [&](const Blocks& o, uint32_t m, const float* val) {
                    float step, inv;
                    block_step(m, &step, &inv);
                    uint32_t w[16];
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        w[q] = e4m3x4(__fmul_rn(val[4 * q], inv), __fmul_rn(val[4 * q + 1], inv), __fmul_rn(val[4 * q + 2], inv), __fmul_rn(val[4 * q + 3], inv));
                    if (!live || !ok) return;
                    if (block_nonfinite(m)) note(P.status, SRQ_ERR_NONFINITE);
                    if (egrp == 0) o.scale[row * o.ld_scale + tn] = step;
                    store_codes64(o.codes + row * o.ld, f0, P.N, w);
                };
                if (P.gate.codes || P.up.codes) {
                    uint32_t mg = 0u, mu = 0u;
#pragma unroll
                    for (int i = 0; i < 64; ++i) { mg = max(mg, abs_word(acc[i])); mu = max(mu, abs_word(acc[64 + i])); }
                    T->amax[par][0][egrp][trow] = mg; T->amax[par][1][egrp][trow] = mu;
                    asm volatile("bar.sync 3, 256;" ::: "memory");
                    mg = max(mg, T->amax[par][0][egrp ^ 1][trow]); mu = max(mu, T->amax[par][1][egrp ^ 1][trow]);
                    if (P.gate.codes) emit(P.gate, mg, acc);
                    if (P.up.codes) emit(P.up, mu, acc + 64);
                }
                uint32_t mh = 0u;
                if (P.gelu) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) { acc[i] = act_of<true>(acc[i]) * acc[64 + i]; mh = max(mh, abs_word(acc[i])); }
                } else {
#pragma unroll
                    for (int i = 0; i < 64; ++i) { acc[i] = act_of<false>(acc[i]) * acc[64 + i]; mh = max(mh, abs_word(acc[i])); }
                }
                if (P.out && live && ok) {
                    const bool vec = P.h_vec && f0 + 64 <= P.N;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        if (P.out_bf16) store8((__nv_bfloat16*)P.out + row * P.ldo, f0 + 8 * q, P.N, vec, acc + 8 * q);
                        else store8((float*)P.out + row * P.ldo, f0 + 8 * q, P.N, vec, acc + 8 * q);
                    }
                }
                if (P.h.codes) {
                    T->amax[par][2][egrp][trow] = mh;
                    asm volatile("bar.sync 3, 256;" ::: "memory");
                    mh = max(mh, T->amax[par][2][egrp ^ 1][trow]);
                    emit(P.h, mh, acc);
                }
                par ^= 1;            // these words are written again two tiles on, a barrier after everyone has read them
            } else {
                const int32_t wrow = (int32_t)(row0 + quarter * 32);
                const int64_t c_first = col0 + 128 * egrp;
                if (P.tma_out && P.out_bf16) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t w[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = pack_bf16(acc[64 * j + 2 * i], acc[64 * j + 2 * i + 1]);
                        if (lane == 0) bulk_wait_read();
                        __syncwarp();
                        stage_block(stage, lane, w);
                        fence_async_smem();
                        __syncwarp();
                        const int64_t c = c_first + 64 * j;
                        if (lane == 0 && wrow < P.M && c < P.N) { tma_store_2d(&map_out, stage, (int32_t)c, wrow); bulk_commit(); }
                    }
                } else if (P.tma_out) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(acc[32 * j + i]);
                        if (lane == 0) bulk_wait_read();
                        __syncwarp();
                        stage_block(stage, lane, w);
                        fence_async_smem();
                        __syncwarp();
                        const int64_t c = c_first + 32 * j;
                        if (lane == 0 && wrow < P.M && c < P.N) {
                            if (P.accumulate) tma_reduce_add_2d(&map_out, stage, (int32_t)c, wrow);
                            else tma_store_2d(&map_out, stage, (int32_t)c, wrow);
                            bulk_commit();
                        }
                    }
                } else if (row < P.M) {
                    if (P.out_bf16) {
                        __nv_bfloat16* dst = (__nv_bfloat16*)P.out + row * P.ldo;
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (c_first + i < P.N) dst[c_first + i] = __float2bfloat16_rn(acc[i]);
                    } else {
                        float* dst = (float*)P.out + row * P.ldo;
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (c_first + i < P.N) dst[c_first + i] = P.accumulate ? __fadd_rn(dst[c_first + i], acc[i]) : acc[i];
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
};
template <int BN, bool GLU>
struct SmallTail {
    using C = SmallCfg<BN, GLU>;
    uint64_t full[C::STAGES], empty[C::STAGES], tmem_full[C::BUFS], tmem_empty[C::BUFS], drain;
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    alignas(16) float token_scale[4][4][BN];           // [warp][k-block of the chunk][token]
};
constexpr int SMALL_THREADS = 192;
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
__global__ void __launch_bounds__(SMALL_THREADS, 1)
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
        for (int b = 0; b < BUFS; ++b) { mbar_init(&T->tmem_full[b], 1); mbar_init(&T->tmem_empty[b], 4); }
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
        if (lane == 0) {
            const uint32_t idesc = make_idesc(1, 128, BN);
            uint32_t it = 0;
            bool ok = true;
            for (int32_t kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u, buf = it % BUFS, use = it / BUFS;
                if (!mbar_wait(&T->tmem_empty[buf], (use & 1u) ^ 1u, &T->abort_flag) ||
                    !mbar_wait(&T->full[s], ph, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; break; }
                tc_fence_after();
                const uint64_t dw = make_smem_desc(smem_u32(smem + (size_t)s * C::STAGE_BYTES));
                const uint64_t dx = dw + (uint64_t)((C::W_BYTES * (GLU ? 2 : 1)) >> 4);
                const uint32_t d = tmem_base + buf * C::COLS;
#pragma unroll
                for (int k = 0; k < GB_K / GB_UMMA_K; ++k) {
                    const uint64_t o = (uint64_t)((k * GB_UMMA_K) >> 4);
                    umma<1, 1>(d, dw + o, dx + o, idesc, k ? 1u : 0u);
                    if constexpr (GLU) umma<1, 1>(d + BN, dw + (uint64_t)(C::W_BYTES >> 4) + o, dx + o, idesc, k ? 1u : 0u);
                }
                umma_commit<1>(&T->empty[s], false);
                umma_commit<1>(&T->tmem_full[buf], false);
            }
            if (!ok) {
                umma_commit<1>(&T->drain, false);
                const uint64_t w0 = global_ns();
                while (!mbar_try_wait(&T->drain, 0u) && global_ns() - w0 < WAIT_LIMIT_NS) {}
            }
        }
    } else {
        const int quarter = warp & 3, ew = warp - 2;
        const int wrow = quarter * 32 + lane;              // weight row within the tile = TMEM lane
        const int64_t n = n0 + wrow;
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
        const float* rw = n < P.N ? P.b.scale + (P.b.tile_rows > 1 ? tn : n) * P.b.ld_scale : nullptr;
        const float* rw2 = GLU && n < P.N ? P.b2.scale + (P.b2.tile_rows > 1 ? tn : n) * P.b2.ld_scale : nullptr;
        constexpr int TPL = (BN + 31) / 32;                // tokens whose step sizes this lane fetches
        const float* rt[TPL];
#pragma unroll
        for (int i = 0; i < TPL; ++i) {
            const int64_t t = t0 + lane + 32 * i;
            rt[i] = (lane + 32 * i < BN && t < P.M) ? P.a.scale + (P.a.tile_rows > 1 ? t / QBLK : t) * P.a.ld_scale : nullptr;
        }
        float (*ts)[BN] = T->token_scale[ew];
        float acc[C::COLS];
#pragma unroll
        for (int i = 0; i < C::COLS; ++i) acc[i] = 0.0f;
        bool ok = true;
        float4 nw = scales4(rw, kb0 >> 2, P.num_kb, P.b_vec), nw2 = scales4(rw2, kb0 >> 2, P.num_kb, P.b_vec);
        float4 nt[TPL];
#pragma unroll
        for (int i = 0; i < TPL; ++i) nt[i] = scales4(rt[i], kb0 >> 2, P.num_kb, P.a_vec);
        float4 cw = nw, cw2 = nw2;
        uint32_t it = 0;
#pragma unroll 1
        for (int32_t kb = kb0; kb < kb1; ++kb, ++it) {
            const int32_t in4 = kb & 3;
            if (in4 == 0 || kb == kb0) {
                cw = nw; cw2 = nw2;
                __syncwarp();                              // the previous chunk has been read
#pragma unroll
                for (int i = 0; i < TPL; ++i) {
                    const int t = lane + 32 * i;
                    if (t < BN) { ts[0][t] = nt[i].x; ts[1][t] = nt[i].y; ts[2][t] = nt[i].z; ts[3][t] = nt[i].w; }
                }
                __syncwarp();
                const int32_t next = (kb >> 2) + 1;
                nw = scales4(rw, next, P.num_kb, P.b_vec);
                if constexpr (GLU) nw2 = scales4(rw2, next, P.num_kb, P.b_vec);
#pragma unroll
                for (int i = 0; i < TPL; ++i) nt[i] = scales4(rt[i], next, P.num_kb, P.a_vec);
            }
            const float sw = pick4(cw, in4), sw2 = pick4(cw2, in4);
            const uint32_t buf = it % BUFS, use = it / BUFS;
            if (ok && !mbar_wait(&T->tmem_full[buf], use & 1u, &T->abort_flag)) { gb_give_up(&T->abort_flag, P.status); ok = false; }
            if (__any_sync(0xFFFFFFFFu, !ok)) ok = false;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < C::COLS / 16; ++c) {
                uint32_t v[16];
                tmem_ld16(taddr + buf * C::COLS + 16 * c, v);
                tmem_ready(v);
                const float s = GLU && c >= BN / 16 ? sw2 : sw;
                const float* tk = &ts[in4][(16 * c) % BN];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 f = *reinterpret_cast<const float4*>(tk + 4 * q);
                    acc[16 * c + 4 * q + 0] = fmaf(__uint_as_float(v[4 * q + 0]), s * f.x, acc[16 * c + 4 * q + 0]);
                    acc[16 * c + 4 * q + 1] = fmaf(__uint_as_float(v[4 * q + 1]), s * f.y, acc[16 * c + 4 * q + 1]);
                    acc[16 * c + 4 * q + 2] = fmaf(__uint_as_float(v[4 * q + 2]), s * f.z, acc[16 * c + 4 * q + 2]);
                    acc[16 * c + 4 * q + 3] = fmaf(__uint_as_float(v[4 * q + 3]), s * f.w, acc[16 * c + 4 * q + 3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&T->tmem_empty[buf]);
        }
        // this CTA's part of every sum: [token (gate, then up)][weight row], in the ring, which nothing uses any more
        float* part = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int i = 0; i < C::COLS; ++i) part[i * 128 + wrow] = acc[i];
    }

    __syncwarp();
    tc_fence_before();
    cluster_sync();                      // all parts are there
    if (warp >= 2) {
        // token t of the tile belongs to CTA t % parts and to one of its warps; a lane takes four columns
        const int64_t c = n0 + 4 * lane;
        const uint32_t base = smem_u32(smem) + (uint32_t)lane * 16u;
        for (int t = (int)rank + (int)parts * (warp - 2); t < BN && t0 + t < P.M; t += (int)parts * 4) {
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f}, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (uint32_t r = 0; r < parts; ++r) {
                const float4 f = ld_cluster_f4(map_to_cta(base + (uint32_t)t * 512u, r));
                x[0] += f.x; x[1] += f.y; x[2] += f.z; x[3] += f.w;
                if constexpr (GLU) {
                    const float4 h = ld_cluster_f4(map_to_cta(base + (uint32_t)(BN + t) * 512u, r));
                    y[0] += h.x; y[1] += h.y; y[2] += h.z; y[3] += h.w;
                }
            }
            const int64_t row = t0 + t;
            if constexpr (GLU) {
                auto emit = [&](const Blocks& o, const float (&val)[4]) {
                    uint32_t m = max(max(abs_word(val[0]), abs_word(val[1])), max(abs_word(val[2]), abs_word(val[3])));
                    m = __reduce_max_sync(0xFFFFFFFFu, m);
                    float step, inv;
                    block_step(m, &step, &inv);
                    if (lane == 0) {
                        o.scale[row * o.ld_scale + tn] = step;
                        if (block_nonfinite(m)) note(P.status, SRQ_ERR_NONFINITE);
                    }
                    const uint32_t w = e4m3x4(__fmul_rn(val[0], inv), __fmul_rn(val[1], inv), __fmul_rn(val[2], inv), __fmul_rn(val[3], inv));
                    uint8_t* dst = o.codes + row * o.ld + c;
                    if (c + 4 <= P.N) *reinterpret_cast<uint32_t*>(dst) = w;
                    else
                        for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = (uint8_t)(w >> (8 * e));
                };
                if (P.gate.codes) emit(P.gate, x);
                if (P.up.codes) emit(P.up, y);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (P.gelu ? act_of<true>(x[e]) : act_of<false>(x[e])) * y[e];
                if (P.h.codes) emit(P.h, x);
            }
            if (P.out) {
                if (P.out_bf16) {
                    __nv_bfloat16* dst = (__nv_bfloat16*)P.out + row * P.ldo + c;
                    if (P.h_vec && c + 4 <= P.N) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                    else
                        for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = __float2bfloat16_rn(x[e]);
                } else {
                    float* dst = (float*)P.out + row * P.ldo + c;
                    if (P.accumulate)
                        for (int e = 0; e < 4; ++e) if (c + e < P.N) x[e] = __fadd_rn(dst[e], x[e]);
                    if (P.h_vec && c + 4 <= P.N) *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
                    else
                        for (int e = 0; e < 4; ++e) if (c + e < P.N) dst[e] = x[e];
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
static bool encode_result(CUtensorMap* map, void* base, bool bf16, int64_t rows, int64_t cols, int64_t ld) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const unsigned esize = bf16 ? 2 : 4;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * esize};
    cuuint32_t box[2] = {128 / esize, 32};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
            cfg.gridDim = dim3((unsigned)(d.sms / s * s)); cfg.blockDim = dim3(SMALL_THREADS); cfg.dynamicSmemBytes = small_smem<16, false>();
            if (cudaOccupancyMaxActiveClusters(&n, gemm_blocks_small_kernel<16, false>, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
            d.clusters[s] = n;
        }
        d.ready = true;
    }
    *out = &d;
    return true;
}

// In how many parts the contraction of `tiles` few-token tiles is cut: the split with the fewest k-blocks
// per SM, counting whole rounds of resident clusters; ties go to fewer parts.
static int small_parts(const BlocksDevice& d, int64_t tiles, int32_t num_kb) {
    int best = 1;
    int64_t best_cost = -1;
    for (int s = 1; s <= 8 && s <= num_kb; ++s) {
        if (d.clusters[s] <= 0) continue;
        const int32_t per = (num_kb + s - 1) / s;
        if ((num_kb + per - 1) / per != s) continue;                 // a part would be empty
        const int64_t rounds = (tiles + d.clusters[s] - 1) / d.clusters[s];
        const int64_t cost = rounds * (per + 4);                     // a round costs about four k-blocks on top
        if (best_cost < 0 || cost < best_cost) { best = s; best_cost = cost; }
    }
    return best;
}

static bool scale_vec(const Blocks& b) { return (uintptr_t)b.scale % 16 == 0 && b.ld_scale % 4 == 0; }

template <int BN, bool GLU>
static cudaError_t launch_small_bn(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mb2, const GemmBlocksParams& P,
                                   int parts, int64_t tiles_n, int64_t tiles_t, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles_n * parts), (unsigned)tiles_t); cfg.blockDim = dim3(SMALL_THREADS);
    cfg.dynamicSmemBytes = small_smem<BN, GLU>(); cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = (unsigned)parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = pdl_allowed(stream) ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_blocks_small_kernel<BN, GLU>, ma, mb, mb2, P);
}

template <bool GLU, bool COLV>
static cudaError_t launch_pair(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mb2, const CUtensorMap& mo,
                               const GemmBlocksParams& P, unsigned pairs, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pairs * 2); cfg.blockDim = dim3(GB_THREADS); cfg.dynamicSmemBytes = gb_smem(); cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = pdl_allowed(stream) ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_blocks_kernel<GLU, COLV>, ma, mb, mb2, mo, P);
}

// Few-token form: as many tokens per CTA as cover M, 128 at most (64 in the gated block, whose sums are two).
static srq_status_t run_small(const BlocksDevice& d, GemmBlocksParams& P, bool glu, int64_t Kc, cudaStream_t stream) {
    int bn = 16;
    while (bn < P.M && bn < (glu ? 64 : 128)) bn *= 2;
    const int64_t tiles_n = (P.N + 127) / 128, tiles_t = (P.M + bn - 1) / bn;
    const int parts = small_parts(d, tiles_n * tiles_t, P.num_kb);
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

static srq_status_t run_pairs(const BlocksDevice& d, GemmBlocksParams& P, bool glu, int64_t Kc, cudaStream_t stream) {
    if (d.pairs <= 0) return SRQ_ERR_UNSUPPORTED;
    P.tiles_m = (int32_t)((P.M + 2 * GB_M - 1) / (2 * GB_M));
    P.tiles_n = (int32_t)((P.N + (glu ? 128 : GB_N) - 1) / (glu ? 128 : GB_N));
    CUtensorMap ma, mb, mb2, mo;
    if (!encode_codes(&ma, P.a, P.M, Kc, GB_M) || !encode_codes(&mb, P.b, P.N, Kc, 128)) return SRQ_ERR_CUDA;
    mb2 = mb; mo = mb;
    if (glu && !encode_codes(&mb2, P.b2, P.N, Kc, 128)) return SRQ_ERR_CUDA;
    const int per16 = P.out_bf16 ? 8 : 4;
    const bool out16 = P.out && (uintptr_t)P.out % 16 == 0 && P.ldo % per16 == 0;
    P.h_vec = out16;
    // a row must also end on a 16-byte boundary: a block store that reaches over the map's edge may write the whole
    // last 16-byte piece
    P.tma_out = !glu && out16 && P.N % per16 == 0 && encode_result(&mo, P.out, P.out_bf16, P.M, P.N, P.ldo);
    const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n;
    const unsigned pairs = (unsigned)(tiles < d.pairs ? tiles : d.pairs);
    const bool colv = P.b.tile_rows == 1;
    cudaError_t e;
    if (glu) e = colv ? launch_pair<true, true>(ma, mb, mb2, mo, P, pairs, stream) : launch_pair<true, false>(ma, mb, mb2, mo, P, pairs, stream);
    else e = colv ? launch_pair<false, true>(ma, mb, mb2, mo, P, pairs, stream) : launch_pair<false, false>(ma, mb, mb2, mo, P, pairs, stream);
    count_launch();
    return e == cudaSuccess ? SRQ_OK : SRQ_ERR_CUDA;
}

// Few-token kernel or CTA pairs.
static bool use_small(const BlocksDevice& d, const GemmBlocksParams& P, bool glu) {
    (void)d; (void)glu;
    return P.M <= 128;
}

srq_status_t launch_gemm_blocks(const GemmBlocksArgs& g, uint32_t* status, cudaStream_t stream) {
    BlocksDevice* d = nullptr;
    if (!blocks_device(&d)) return SRQ_ERR_CUDA;
    GemmBlocksParams P = {};
    P.M = g.M; P.N = g.N; P.num_kb = (int32_t)((g.Kc + GB_K - 1) / GB_K);
    P.a = g.a; P.b = g.b; P.a_vec = scale_vec(g.a); P.b_vec = scale_vec(g.b);
    P.out = g.out; P.ldo = g.ldo; P.out_bf16 = g.out_dt == SRQ_BF16; P.accumulate = g.accumulate;
    P.status = status;
    return use_small(*d, P, false) ? run_small(*d, P, false, g.Kc, stream) : run_pairs(*d, P, false, g.Kc, stream);
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
    return use_small(*d, P, true) ? run_small(*d, P, true, g.K, stream) : run_pairs(*d, P, true, g.K, stream);
}

}  // namespace srq
