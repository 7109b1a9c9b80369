// Products with a quantized layer for many rows of x: y = act(x What^T + bias) + residual
// on the fifth-generation tensor cores.
//
// A CTA takes 128 outputs and BN rows of x: y^T[128 x BN] = (c - z)[128 x p] x^T, 64 columns
// a step.  Bound by the tensor cores.  Roles:
//   warp 0         brings x's tiles by TMA (128-byte swizzle; columns past p and rows past
//                  the last are filled with zeros);
//   warp 1         issues the products, accumulators in tensor memory;
//   warp 2         brings codes by bulk copies, some steps ahead, into a ring of their own;
//   warps 4-11     turn codes into the other operand: a pair of codes becomes 16-bit floats
//                  c - z (exact), and 16-byte pieces go to shared memory in the same swizzle.  Four
//                  warps take the even steps and four the odd ones, two row tiles of 16 outputs
//                  each, so that a step's chain of reading, turning and writing has two steps' time;
//   warps 12-19    fold accumulators into registers, times the scale: at the end of each
//                  group, or every kSegment columns with one grid a row (the tensor cores'
//                  accumulators lose up to a unit in the last place with each addition, a
//                  short chain's worth of which binary32 does not show).  Two accumulators take turns.
// Where there are few tiles the CTAs of a cluster share a tile's columns; their sums meet in shared
// memory in order.  Results leave through shared memory, so that rows of y are written 16 bytes a lane.
#pragma once

#include <cooperative_groups.h>

#include <atomic>

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
    static constexpr int A_BYTES = kTileOut * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 6 : 7;
    static constexpr int HALF = BN / 2;    // columns of a folding thread
    static constexpr int CODE_RING = 32 * 1024;
    static constexpr int SMEM = STAGES * STAGE + CODE_RING + 1024 + 512;
    // registers a thread: 96 at launch, dealt out anew by role (warps 0-3, two warpgroups that turn, two that fold)
    static constexpr int FOLD_REGS = BN == 256 ? 168 : BN == 128 ? 120 : 96, TURN_REGS = BN == 256 ? 56 : BN == 128 ? 80 : 96,
                         LEAD_REGS = BN == 256 ? 32 : BN == 128 ? 80 : 96;
    static_assert(2 * FOLD_REGS + 2 * TURN_REGS + LEAD_REGS <= 5 * 96, "as many as the block was launched with");
    static_assert(BN * kTileOut * 4 <= STAGES * STAGE, "results fit the ring");
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

// A wait that reads the clock only when it takes long.
__device__ __forceinline__ bool wait_on(uint64_t *bar, uint32_t parity, volatile int *abort) {
    for (int n = 0; n < 16; ++n)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_bounded(bar, parity, abort);
}
__device__ __forceinline__ bool wait_warp_on(uint64_t *bar, uint32_t parity, volatile int *abort) {
    return __all_sync(0xffffffffu, wait_on(bar, parity, abort)) != 0;
}

__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int B, int BN, bool HALF>
__global__ void __launch_bounds__(kTileThreads, 1) k_linear_tiles(const LinearArgs a, const __grid_constant__ CUtensorMap xmap) {
    using F = TilesOf<BN>;
    using TU = Turn<B, HALF>;
    extern __shared__ uint8_t raw_smem[];
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);
    constexpr int CODES = 8 * 128 * B, CODE_STAGES = F::CODE_RING / CODES;   // bytes of a step's codes
    uint8_t *code_ring = smem + F::STAGES * F::STAGE;
    uint64_t *full = reinterpret_cast<uint64_t *>(code_ring + F::CODE_RING);
    uint64_t *empty = full + F::STAGES, *acc_full = empty + F::STAGES, *acc_empty = acc_full + 2, *drain = acc_empty + 2;
    uint64_t *code_full = drain + 1, *code_empty = code_full + CODE_STAGES;
    static_assert((2 * F::STAGES + 5 + 2 * CODE_STAGES) * 8 + 8 <= 512, "room for the barriers");
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(code_empty + CODE_STAGES);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int out_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(ranks));
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * BN;
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
    if (warp == 0 && lane == 0) prefetch_tensormap(&xmap);
    if (warp == 1) tmem_alloc(tmem_slot, 2 * BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto give_up = [&]() {
        *abort_flag = 1;
        set_error(a.err, ERR_TIMEOUT);
    };

    // all threads: sums are in place; and nobody leaves while they are read
    auto meet = [&]() {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };

    if (warp < kTurnWarp) {
        if constexpr (F::LEAD_REGS < 96) fewer_registers<F::LEAD_REGS>();
    }
    if (warp == 0) {
        if (lane == 0) {
            int n = 0;
            for (int u = begin; u < end; ++u, ++n) {
                const int s = n % F::STAGES;
                if (!wait_on(&empty[s], ((n / F::STAGES) & 1u) ^ 1u, abort_flag)) {
                    give_up();
                    break;
                }
                mbar_arrive_expect_tx(&full[s], F::B_BYTES);
                tma_load_2d(&xmap, smem + s * F::STAGE + F::A_BYTES, &full[s], u * kUnitCols, static_cast<int>(m0));
            }
            // the last copy into each stage has landed before the CTA goes on (after a wait that gave up the other
            // arrivals may be missing: then the time limit ends the wait, long after the copy has landed)
            for (int k = n > F::STAGES ? n - F::STAGES : 0; k < n; ++k) mbar_wait_bounded(&full[k % F::STAGES], (k / F::STAGES) & 1u, nullptr);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = HALF ? idesc_f16_f32(kTileOut, BN) : idesc_bf16_f32(kTileOut, BN);
            int n = 0, c = 0;
            bool ok = true;
            for (int u = begin; ok && u < end; ++c) {
                const int buf = c & 1;
                if (c >= 2 && !wait_on(&acc_empty[buf], ((c >> 1) - 1) & 1u, abort_flag)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t dst = tmem + static_cast<uint32_t>(buf * BN);
                const int upto = min((u / seg + 1) * seg, end);
                for (int first = 1; u < upto; ++u, ++n, first = 0) {
                    const int s = n % F::STAGES;
                    if (!wait_on(&full[s], (n / F::STAGES) & 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t at = smem_u32(smem + s * F::STAGE);
                    const uint64_t da = smem_desc_k128(at), db = smem_desc_k128(at + F::A_BYTES);
#pragma unroll
                    for (int k = 0; k < kUnitCols / 16; ++k) mma_bf16_ss(dst, da + 2u * k, db + 2u * k, idesc, first && k == 0 ? 0u : 1u);
                    mma_commit(&empty[s]);
                }
                if (ok) mma_commit(&acc_full[buf]);
            }
            if (!ok) give_up();
            mma_commit(drain);                            // nothing is in flight when tensor memory is freed
            mbar_wait_bounded(drain, 0u, nullptr);
        }
    } else if (warp == 2) {
        // lanes 0 .. 7 copy a row tile's unit each (tiles that are not there repeat the last one; their results go nowhere)
        const int64_t row_tile = min(out_tile * (kTileOut / kTileRows) + (lane & 7), a.g.row_tiles - 1);
        const uint8_t *code = a.g.codes + (row_tile * a.g.units + begin) * (128 * B);
        int n = 0;
        for (; n < end - begin; ++n) {
            const int s = n % CODE_STAGES;
            if (!wait_warp_on(&code_empty[s], ((n / CODE_STAGES) & 1u) ^ 1u, abort_flag)) {
                if (lane == 0) give_up();
                break;
            }
            if (lane == 0) mbar_arrive_expect_tx(&code_full[s], CODES);
            __syncwarp();
            if (lane < 8) bulk_load(code_ring + s * CODES + lane * (128 * B), code + static_cast<int64_t>(n) * (128 * B), 128 * B, &code_full[s]);
        }
        if (lane == 0)
            for (int k = n > CODE_STAGES ? n - CODE_STAGES : 0; k < n; ++k)
                mbar_wait_bounded(&code_full[k % CODE_STAGES], (k / CODE_STAGES) & 1u, nullptr);
    } else if (warp >= kTurnWarp && warp < kFoldWarp) {
        if constexpr (F::TURN_REGS < 96) fewer_registers<F::TURN_REGS>();
        const int r = lane >> 2, t = lane & 3, sub = 2 * ((warp - kTurnWarp) & 3), odd_steps = (warp - kTurnWarp) >> 2;
        uint32_t zero[2][2][TU::LEVELS];
        const uint8_t *zeros[2];                          // of row r of either row tile; row r + 8's 8 behind
#pragma unroll
        for (int i = 0; i < 2; ++i)
            zeros[i] = a.g.zeros + static_cast<int64_t>(min(out_tile * (kTileOut / kTileRows) + sub + i, a.g.row_tiles - 1)) * a.g.groups * kTileRows + r;
        // the two pieces of a row that a lane has (chunks 0 and 1) are written odd rows' second one first: so the eight
        // lanes of a phase write to all banks
        const int odd = r & 1;
        const int row_at = (sub * kTileRows + r) * 128, piece0 = row_at + (((4 * odd + t) ^ (r & 7)) << 4), piece1 = row_at + (((4 - 4 * odd + t) ^ (r & 7)) << 4);
        int next_grid = begin;
        bool ok = true;
        for (int n = odd_steps; ok && n < end - begin; n += 2) {
            const int u = begin + n;
            if (u >= next_grid) {
                const int g = a.g.groups > 1 ? u / a.g.group_units : 0;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) TU::zero(static_cast<float>(zeros[i][g * kTileRows + 8 * h]), zero[i][h]);
                next_grid = (g + 1) * a.g.group_units;
            }
            const int cs = n % CODE_STAGES, s = n % F::STAGES;
            ok = wait_warp_on(&code_full[cs], (n / CODE_STAGES) & 1u, abort_flag);
            if (!ok) break;
            uint32_t w[2][B];
#pragma unroll
            for (int i = 0; i < 2; ++i) read_unit<B>(code_ring + cs * CODES + (sub + i) * (128 * B), lane, w[i]);
            __syncwarp();
            if (lane == 0) mbar_arrive(&code_empty[cs]);
            ok = wait_warp_on(&empty[s], ((n / F::STAGES) & 1u) ^ 1u, abort_flag);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t v[2][2][4];
                TU::unit(w[i], zero[i], v);
                uint8_t *to = smem + s * F::STAGE + i * (kTileRows * 128);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t q[2][4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        q[0][p] = odd ? v[1][h][p] : v[0][h][p];
                        q[1][p] = odd ? v[0][h][p] : v[1][h][p];
                    }
                    *reinterpret_cast<uint4 *>(to + piece0 + h * 1024) = make_uint4(q[0][0], q[0][1], q[0][2], q[0][3]);
                    *reinterpret_cast<uint4 *>(to + piece1 + h * 1024) = make_uint4(q[1][0], q[1][1], q[1][2], q[1][3]);
                }
            }
            fence_to_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&full[s]);
        }
        if (!ok && lane == 0) give_up();
    } else if (warp >= kFoldWarp) {
        if constexpr (F::FOLD_REGS > 96) more_registers<F::FOLD_REGS>();
        const int quad = warp & 3, side = (warp - kFoldWarp) >> 2;
        const int row = quad * 32 + lane, tile = out_tile * (kTileOut / kTileRows) + row / kTileRows;
        const int64_t row_tile = min(tile, a.g.row_tiles - 1);
        const uint32_t from = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(side * F::HALF);
        float acc[F::HALF];
#pragma unroll
        for (int i = 0; i < F::HALF; ++i) acc[i] = 0.0f;
        bool ok = true;
        int c = 0;
        for (int u = begin; u < end; ++c) {
            const int buf = c & 1, g = a.g.groups > 1 ? u / a.g.group_units : 0;
            const float scale = a.g.scales[(row_tile * a.g.groups + g) * kTileRows + row % kTileRows];
            ok = wait_warp_on(&acc_full[buf], (c >> 1) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int q = 0; q < F::HALF / 16; ++q) {
                float v[16];
                tmem_ld_16(from + static_cast<uint32_t>(buf * BN + q * 16), v);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[q * 16 + i] = fmaf(scale, v[i], acc[q * 16 + i]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);
            u = min((u / seg + 1) * seg, end);
        }
        if (!ok && lane == 0) give_up();
        // every product has been taken: the ring is free for the sums, [row of x][output]
        float *sums = reinterpret_cast<float *>(smem);
        if (ok)
#pragma unroll
            for (int i = 0; i < F::HALF; ++i) sums[(side * F::HALF + i) * kTileOut + row] = acc[i];
    }
    if (warp < kFoldWarp) {
        tc_fence_before();
        meet();
        if (warp == 1) tmem_dealloc(tmem, 2 * BN);
        meet();
        return;
    }
    tc_fence_before();
    meet();
    // ---- out: eight outputs of a row of x a thread; the cluster's CTAs take rows in turn ----
    const int64_t out0 = static_cast<int64_t>(out_tile) * kTileOut;
    const float *sums = reinterpret_cast<const float *>(smem);
    const int failed = *abort_flag;
    for (int e = threadIdx.x - 32 * kFoldWarp; e < BN * (kTileOut / 8) && !failed; e += 256) {
        const int tok = e / (kTileOut / 8), o = 8 * (e % (kTileOut / 8));
        const int64_t m = m0 + tok, i = out0 + o;
        if (m >= a.rows || i >= a.g.q || (ranks > 1 && tok % ranks != rank)) continue;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.0f;
        for (int q = 0; q < ranks; ++q) {
            const float4 *p = reinterpret_cast<const float4 *>((ranks > 1 ? cluster.map_shared_rank(sums, q) : sums) + tok * kTileOut + o);
            const float4 x = p[0], y = p[1];
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        finish_eight(a, v, m, i);
    }
    meet();
}

template <int B, int BN, bool HALF>
cudaError_t launch_tiles_as(const LinearArgs &a, cudaStream_t s) {
    using F = TilesOf<BN>;
    CUtensorMap map;
    if (!(HALF ? make_tmap_f16 : make_tmap_bf16)(&map, a.x, static_cast<uint64_t>(a.rows), static_cast<uint64_t>(a.g.p),
                                                 static_cast<uint64_t>(a.ldx), BN))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> raised{0};
    const void *kernel = reinterpret_cast<const void *>(k_linear_tiles<B, BN, HALF>);
    cudaError_t e = raise_limit(kernel, F::SMEM, raised);
    if (e != cudaSuccess) return e;
    const int64_t tiles = ceil_div(a.g.q, kTileOut), blocks = ceil_div(a.rows, BN);
    int ranks = 1;
    while (ranks < 8 && tiles * blocks * ranks * 2 <= 152 && a.g.units >= 8 * ranks) ranks *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * ranks), static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kTileThreads);
    cfg.dynamicSmemBytes = F::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(ranks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_linear_tiles<B, BN, HALF>, a, map);
}

template <int B, int BN>
cudaError_t launch_tiles_type(const LinearArgs &a, cudaStream_t s) {
    return a.half ? launch_tiles_as<B, BN, true>(a, s) : launch_tiles_as<B, BN, false>(a, s);
}

template <int B>
cudaError_t launch_tiles_bits(const LinearArgs &a, cudaStream_t s) {
    if (a.rows <= 64) return launch_tiles_type<B, 64>(a, s);
    if (a.rows <= 128) return launch_tiles_type<B, 128>(a, s);
    return launch_tiles_type<B, 256>(a, s);
}

}  // namespace
}  // namespace qe
