// Products with a quantized layer for many rows of x: y = act(x What^T + bias) + residual
// on the fifth-generation tensor cores.
//
// A tile is 128 outputs and BN rows of x: y^T[128 x BN] = (c - z)[128 x p] x^T, 64 columns
// a step.  Bound by the tensor cores and, nearly as much, by shared memory's bandwidth: so
// the turned codes do not pass through it but lie in tensor memory, from where the
// products take their first operand.  Roles:
//   warp 0         brings x's tiles by TMA (128-byte swizzle; columns past p and rows past
//                  the last are filled with zeros);
//   warp 1         issues the products, accumulators in tensor memory;
//   warp 2         brings codes by TMA, some steps ahead, into a ring of their own (one copy a
//                  step: eight bulk copies, a row tile's unit each, took longer to issue);
//   warps 4-11     turn codes into the operand: a pair of codes becomes 16-bit floats c - z
//                  (exact).  Four warps take the even steps and four the odd ones, the two row
//                  tiles of 16 outputs that stand in a warp's 32 lanes of tensor memory;
//   warps 12-19    fold accumulators into registers, times the scale: at the end of each
//                  group, or every kSegment columns with one grid a row (the tensor cores'
//                  accumulators lose up to a unit in the last place with each addition, a
//                  short chain's worth of which binary32 does not show).  Two accumulators take
//                  turns.  Finished tiles leave through shared memory, 16 bytes a lane.
// A CTA takes tile after tile, the next one's products running while the last one leaves.
// Where there are few tiles the CTAs of a cluster share a tile's columns; their sums meet in
// shared memory in order.
#pragma once

#include <cooperative_groups.h>

#include "qe_internal.h"
#include "qe_linear.cuh"

namespace qe {
namespace {

constexpr int kTileOut = 128;
constexpr int kSegmentUnits = 32;          // 2048 columns
constexpr int kTileThreads = 640;
constexpr int kTurnWarp = 4, kFoldWarp = 12;

template <int BN>
struct TilesOf {
    static constexpr int STAGE = BN * 128, STAGES = BN == 192 ? 4 : BN == 128 ? 6 : 8;   // of x, and of turned codes:
    static constexpr int A_COLS = kUnitCols / 2;                                         // these behind the two accumulators
    static constexpr int HALF = BN / 2;    // columns of a folding thread
    static constexpr int OUT_COLS = BN == 64 ? 32 : HALF / 2;                            // that leave at once
    static constexpr int CODE_RING = 32 * 1024, OUT_BYTES = 8 * OUT_COLS * 32 * 4;
    static constexpr int SMEM = STAGES * STAGE + CODE_RING + OUT_BYTES + 1024 + 768;
    // registers a thread: 96 at launch, dealt out anew by role (warps 0-3, two warpgroups that turn, two that fold)
    static constexpr int FOLD_REGS = BN == 192 ? 144 : 96, TURN_REGS = BN == 192 ? 72 : 96, LEAD_REGS = BN == 192 ? 48 : 96;
    static_assert(2 * FOLD_REGS + 2 * TURN_REGS + LEAD_REGS <= 5 * 96, "as many as the block was launched with");
    static_assert(2 * BN + STAGES * A_COLS <= 512, "tensor memory");
    static_assert(BN * kTileOut * 4 <= STAGES * STAGE, "a cluster's sums fit the ring");
    static_assert(SMEM <= 232448, "shared memory");
};

template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// 32 lanes x 16 neighbouring 32-bit columns of tensor memory.
__device__ __forceinline__ void tmem_ld_16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// A row tile's unit, 16 lanes x 32 columns: register 2 j + h of lane 4 r + t goes to lane r + 8 h, column 4 j + t.
__device__ __forceinline__ void tmem_st_unit(uint32_t taddr, const uint32_t (&v)[2][2][4]) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(v[0][0][0]), "r"(v[0][1][0]), "r"(v[0][0][1]), "r"(v[0][1][1]), "r"(v[0][0][2]), "r"(v[0][1][2]), "r"(v[0][0][3]), "r"(v[0][1][3]),
        "r"(v[1][0][0]), "r"(v[1][1][0]), "r"(v[1][0][1]), "r"(v[1][1][1]), "r"(v[1][0][2]), "r"(v[1][1][2]), "r"(v[1][0][3]), "r"(v[1][1][3])
        : "memory");
}

// D += A B with A in tensor memory; and an arrival on a barrier once all products so far have been taken.  Issued by one
// elected lane of a warp that goes along together, so that addresses stay in uniform registers (a step's issue took 411
// cycles from a lane by itself).
__device__ __forceinline__ void mma_ts_one(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(bar)
        : "memory");
}

// A wait that reads the clock only when it takes long.
__device__ __forceinline__ bool wait_on(uint64_t *bar, uint32_t parity, volatile int *abort) {
    for (int n = 0; n < 16; ++n)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_bounded(bar, parity, abort);
}
__device__ __forceinline__ bool wait_warp_on(uint64_t *bar, uint32_t parity, volatile int *abort) {
    return __all_sync(0xffffffffu, wait_on(bar, parity, abort)) != 0;
}

// A place in a ring of N stages.
template <int N>
struct Turnstile {
    int s = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++s == N) {
            s = 0;
            phase ^= 1u;
        }
    }
};

template <int B, int BN, bool HALF>
__global__ void __launch_bounds__(kTileThreads, 1) k_linear_tiles(const LinearArgs a, const __grid_constant__ CUtensorMap xmap,
                                                                  const __grid_constant__ CUtensorMap cmap) {
    using F = TilesOf<BN>;
    using TU = Turn<B, HALF>;
    constexpr int CODES = 8 * 128 * B, CODE_STAGES = F::CODE_RING / CODES;   // bytes of a step's codes
    extern __shared__ uint8_t raw_smem[];
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);
    uint8_t *code_ring = smem + F::STAGES * F::STAGE;
    float *out_stage = reinterpret_cast<float *>(code_ring + F::CODE_RING);
    uint64_t *full = reinterpret_cast<uint64_t *>(code_ring + F::CODE_RING + F::OUT_BYTES), *empty = full + F::STAGES;
    uint64_t *code_full = empty + F::STAGES, *code_empty = code_full + CODE_STAGES;
    uint64_t *acc_full = code_empty + CODE_STAGES, *acc_empty = acc_full + 2, *drain = acc_empty + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    static_assert((2 * F::STAGES + 5 + 2 * CODE_STAGES) * 8 + 8 <= 768, "room for the barriers");
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // a tile's outputs run fastest; a cluster takes one tile, a CTA by itself every gridDim.x-th
    const int out_tiles = (a.g.row_tiles + 7) / 8;
    const int tiles = out_tiles * static_cast<int>((a.rows + BN - 1) / BN);
    const int first_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(ranks)), tile_step = static_cast<int>(gridDim.x / static_cast<unsigned>(ranks));
    const int begin = static_cast<int>(static_cast<int64_t>(a.g.units) * rank / ranks),
              end = static_cast<int>(static_cast<int64_t>(a.g.units) * (rank + 1) / ranks);
    const int seg = a.g.groups > 1 ? a.g.group_units : kSegmentUnits;

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::STAGES; ++s) {
            mbar_init(&full[s], 1 + 4);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 8);
        }
        for (int s = 0; s < CODE_STAGES; ++s) {
            mbar_init(&code_full[s], 1);
            mbar_init(&code_empty[s], 4);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&xmap);
        prefetch_tensormap(&cmap);
    }
    if (warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto give_up = [&]() {
        *abort_flag = 1;
        set_error(a.err, ERR_TIMEOUT);
    };
    // all threads of the cluster: sums are in place; and nobody leaves while they are read
    auto meet = [&]() {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };

    if (warp < kTurnWarp) {
        if constexpr (F::LEAD_REGS < 96) fewer_registers<F::LEAD_REGS>();
    }
    if (warp == 0) {
        if (lane == 0) {
            Turnstile<F::STAGES> at;
            int64_t n = 0;
            bool ok = true;
            for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
                const int m0 = tile / out_tiles * BN;
                for (int u = begin; u < end; ++u, ++n) {
                    ok = wait_on(&empty[at.s], at.phase ^ 1u, abort_flag);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&full[at.s], F::STAGE);
                    tma_load_2d(&xmap, smem + at.s * F::STAGE, &full[at.s], u * kUnitCols, m0);
                    at.next();
                }
            }
            if (!ok) give_up();
            // the last copy into each stage has landed before the CTA goes on
            for (int64_t k = n > F::STAGES ? n - F::STAGES : 0; k < n; ++k)
                mbar_wait_bounded(&full[k % F::STAGES], static_cast<uint32_t>(k / F::STAGES) & 1u, nullptr);
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = HALF ? idesc_f16_f32(kTileOut, BN) : idesc_bf16_f32(kTileOut, BN);
        const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0), empty0 = smem_u32(empty), acc0 = smem_u32(acc_full);
        const uint64_t x0 = smem_desc_k128(smem_u32(smem));
        Turnstile<F::STAGES> at;
        Turnstile<2> acc;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step)
            for (int u = begin; ok && u < end;) {
                ok = wait_warp_on(&acc_empty[acc.s], acc.phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t dst = t0 + static_cast<uint32_t>(acc.s * BN);
                const int upto = min((u / seg + 1) * seg, end);
                for (uint32_t add = 0u; u < upto; ++u, add = 1u) {
                    ok = wait_warp_on(&full[at.s], at.phase, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t db = x0 + static_cast<uint64_t>(at.s * (F::STAGE / 16));
                    const uint32_t da = t0 + static_cast<uint32_t>(2 * BN + at.s * F::A_COLS);
                    mma_ts_one(dst, da, db, idesc, add);
#pragma unroll
                    for (int k = 1; k < kUnitCols / 16; ++k) mma_ts_one(dst, da + 8u * k, db + 2u * k, idesc, 1u);
                    commit_one(empty0 + 8u * at.s);
                    at.next();
                }
                if (ok) commit_one(acc0 + 8u * acc.s);
                acc.next();
            }
        if (!ok && lane == 0) give_up();
        __syncwarp();
        commit_one(smem_u32(drain));                      // nothing is in flight when tensor memory is freed
        mbar_wait_bounded(drain, 0u, nullptr);
    } else if (warp == 2) {
        if (lane == 0) {                                  // (row tiles past the last are zeros)
            Turnstile<CODE_STAGES> at;
            int64_t n = 0;
            bool ok = true;
            for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
                const int row0 = tile % out_tiles * (kTileOut / kTileRows);
                for (int u = begin; u < end; ++u, ++n) {
                    ok = wait_on(&code_empty[at.s], at.phase ^ 1u, abort_flag);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&code_full[at.s], CODES);
                    tma_load_2d(&cmap, code_ring + at.s * CODES, &code_full[at.s], u * 32 * B, row0);
                    at.next();
                }
            }
            if (!ok) give_up();
            for (int64_t k = n > CODE_STAGES ? n - CODE_STAGES : 0; k < n; ++k)
                mbar_wait_bounded(&code_full[k % CODE_STAGES], static_cast<uint32_t>(k / CODE_STAGES) & 1u, nullptr);
        }
    } else if (warp >= kTurnWarp && warp < kFoldWarp) {
        if constexpr (F::TURN_REGS < 96) fewer_registers<F::TURN_REGS>();
        const int r = lane >> 2, quad = warp & 3, odd = (warp - kTurnWarp) >> 2;
        const uint32_t to = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(2 * BN);
        uint32_t zero[2][2][TU::LEVELS];
        Turnstile<CODE_STAGES> cs;
        Turnstile<F::STAGES> as;
        int n = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            const uint8_t *zeros[2];                      // of row r of either row tile; row r + 8's 8 behind
#pragma unroll
            for (int i = 0; i < 2; ++i)
                zeros[i] = a.g.zeros + static_cast<int64_t>(min(tile % out_tiles * (kTileOut / kTileRows) + 2 * quad + i, a.g.row_tiles - 1)) *
                                           a.g.groups * kTileRows + r;
            int next_grid = begin;
            for (int u = begin; u < end; ++u, ++n, cs.next(), as.next()) {
                if ((n & 1) != odd) continue;
                if (u >= next_grid) {
                    const int g = a.g.groups > 1 ? u / a.g.group_units : 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) TU::zero(static_cast<float>(zeros[i][g * kTileRows + 8 * h]), zero[i][h]);
                    next_grid = (g + 1) * a.g.group_units;
                }
                ok = wait_warp_on(&code_full[cs.s], cs.phase, abort_flag);
                if (!ok) break;
                uint32_t w[2][B], v[2][2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) read_unit<B>(code_ring + cs.s * CODES + (2 * quad + i) * (128 * B), lane, w[i]);
                TU::unit(w[0], zero[0], v);
                ok = wait_warp_on(&empty[as.s], as.phase ^ 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const uint32_t dst = to + static_cast<uint32_t>(as.s * F::A_COLS);
                tmem_st_unit(dst, v);
                TU::unit(w[1], zero[1], v);
                tmem_st_unit(dst + (16u << 16), v);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&code_empty[cs.s]);
                    mbar_arrive(&full[as.s]);
                }
            }
        }
        if (!ok && lane == 0) give_up();
    } else if (warp >= kFoldWarp) {
        if constexpr (F::FOLD_REGS > 96) more_registers<F::FOLD_REGS>();
        const int quad = warp & 3, side = (warp - kFoldWarp) >> 2, row = quad * 32 + lane;
        const uint32_t from = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(side * F::HALF);
        Turnstile<2> buf;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            const int out_tile = tile % out_tiles;
            const int64_t row_tile = min(out_tile * (kTileOut / kTileRows) + row / kTileRows, a.g.row_tiles - 1);
            const int64_t m0 = static_cast<int64_t>(tile / out_tiles) * BN + side * F::HALF, out0 = static_cast<int64_t>(out_tile) * kTileOut;
            float acc[F::HALF];
#pragma unroll
            for (int i = 0; i < F::HALF; ++i) acc[i] = 0.0f;
            for (int u = begin; u < end; buf.next()) {
                const int g = a.g.groups > 1 ? u / a.g.group_units : 0;
                const float scale = a.g.scales[(row_tile * a.g.groups + g) * kTileRows + row % kTileRows];
                ok = wait_warp_on(&acc_full[buf.s], buf.phase, abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < F::HALF / 16; ++q) {
                    float v[16];
                    tmem_ld_16(from + static_cast<uint32_t>(buf.s * BN + q * 16), v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[q * 16 + i] = fmaf(scale, v[i], acc[q * 16 + i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[buf.s]);
                u = min((u / seg + 1) * seg, end);
            }
            if (!ok) break;
            if (ranks > 1) {
                // every product has been taken: x's ring is free for the sums, [row of x][output]
                float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
                for (int i = 0; i < F::HALF; ++i) sums[(side * F::HALF + i) * kTileOut + row] = acc[i];
                continue;
            }
            // out, OUT_COLS rows of x at a time: eight outputs of one a lane
            float *mine = out_stage + (warp - kFoldWarp) * (F::OUT_COLS * 32);
#pragma unroll
            for (int part = 0; part < F::HALF / F::OUT_COLS; ++part) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < F::OUT_COLS; ++i) mine[i * 32 + lane] = acc[part * F::OUT_COLS + i];
                __syncwarp();
                const int64_t o = out0 + quad * 32 + 8 * (lane & 3);
#pragma unroll 1
                for (int i = lane >> 2; i < F::OUT_COLS; i += 8) {
                    const int64_t m = m0 + part * F::OUT_COLS + i;
                    if (m >= a.rows || o >= a.g.q) continue;
                    const float4 *p = reinterpret_cast<const float4 *>(mine + i * 32 + 8 * (lane & 3));
                    const float4 x = p[0], y = p[1];
                    float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                    finish_eight(a, v, m, o);
                }
            }
        }
        if (!ok && lane == 0) give_up();
    }
    if (warp < kFoldWarp) {
        tc_fence_before();
        meet();
        if (warp == 1) tmem_dealloc(tmem, 512);
        meet();
        return;
    }
    tc_fence_before();
    meet();
    if (ranks > 1 && first_tile < tiles) {                // the cluster's CTAs take rows of x in turn
        const int64_t m0 = static_cast<int64_t>(first_tile / out_tiles) * BN, out0 = static_cast<int64_t>(first_tile % out_tiles) * kTileOut;
        const float *sums = reinterpret_cast<const float *>(smem);
        const int failed = *abort_flag;
        for (int e = threadIdx.x - 32 * kFoldWarp; e < BN * (kTileOut / 8) && !failed; e += 256) {
            const int tok = e / (kTileOut / 8), o = 8 * (e % (kTileOut / 8));
            const int64_t m = m0 + tok, i = out0 + o;
            if (m >= a.rows || i >= a.g.q || tok % ranks != rank) continue;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            for (int q = 0; q < ranks; ++q) {
                const float4 *p = reinterpret_cast<const float4 *>(cluster.map_shared_rank(sums, q) + tok * kTileOut + o);
                const float4 x = p[0], y = p[1];
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
            }
            finish_eight(a, v, m, i);
        }
    }
    meet();
}

template <int B, int BN, bool HALF>
cudaError_t launch_tiles_as(const LinearArgs &a, cudaStream_t s) {
    using F = TilesOf<BN>;
    CUtensorMap map, codes;
    if (!(HALF ? make_tmap_f16 : make_tmap_bf16)(&map, a.x, static_cast<uint64_t>(a.rows), static_cast<uint64_t>(a.g.p),
                                                 static_cast<uint64_t>(a.ldx), BN) ||
        !make_tmap_words(&codes, a.g.codes, static_cast<uint64_t>(a.g.row_tiles), static_cast<uint64_t>(a.g.units) * 32 * B, 32 * B, kTileOut / kTileRows))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> raised{0};
    const void *kernel = reinterpret_cast<const void *>(k_linear_tiles<B, BN, HALF>);
    cudaError_t e = raise_limit(kernel, F::SMEM, raised);
    if (e != cudaSuccess) return e;
    const int64_t tiles = ceil_div(a.g.q, kTileOut) * ceil_div(a.rows, BN), sms = linear_sms();
    int ranks = 1;
    while (ranks < 8 && tiles * ranks * 2 <= sms && a.g.units >= 8 * ranks) ranks *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ranks > 1 ? tiles * ranks : tiles < sms ? tiles : sms));
    cfg.blockDim = dim3(kTileThreads);
    cfg.dynamicSmemBytes = F::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(ranks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_linear_tiles<B, BN, HALF>, a, map, codes);
}

template <int B, int BN>
cudaError_t launch_tiles_type(const LinearArgs &a, cudaStream_t s) {
    return a.half ? launch_tiles_as<B, BN, true>(a, s) : launch_tiles_as<B, BN, false>(a, s);
}

template <int B>
cudaError_t launch_tiles_bits(const LinearArgs &a, cudaStream_t s) {
    if (a.rows <= 64) return launch_tiles_type<B, 64>(a, s);
    if (a.rows <= 128) return launch_tiles_type<B, 128>(a, s);
    return launch_tiles_type<B, 192>(a, s);
}

}  // namespace
}  // namespace qe
