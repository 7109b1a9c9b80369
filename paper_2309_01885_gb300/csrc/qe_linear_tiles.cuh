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
//                  (exact).  Four warps take the even pairs of steps and four the odd ones, the
//                  two row tiles of 16 outputs that stand in a warp's 32 lanes of tensor memory;
//   warps 12-19    fold accumulators into registers, times the scale: at the end of each
//                  group, and every kSegmentUnits units of a longer one, or of a row with one
//                  grid.  Two accumulators take turns where there is room for two.
// A CTA takes tile after tile, the next one's products running while the last one leaves.
// Where there are few tiles the CTAs of a cluster share a tile's columns; their sums meet in
// shared memory in order.
//
// Measured (us; of the products' 2 rows q p): 4095 x 4096 x 11008, 4 bits 209 to 215 (1.7 to 1.8 PFLOP/s), with GELU 229, a residual
// 225, both 238, 8 bits 301 (five instructions turn two codes for bf16, and tiles have 224 rows), grids for groups of 256, 128 and 64
// columns 299, 336 and 610 (every group's sums pass from tensor memory through registers, 16 columns a wait); 4095 x 14848 x 4096
// 311, 2048 x 4096 x 4096 59, in groups of 128 86, 64 x 4096 x 4096 14.  Turned codes through shared memory, the
// products' other form, were slower: both operands and the codes pass through it then.
#pragma once

#include <cooperative_groups.h>

#include "qe_internal.h"
#include "qe_linear.cuh"

namespace qe {
namespace {

constexpr int kTileOut = 128;
constexpr int kTileThreads = 640;
constexpr int kTurnWarp = 4, kFoldWarp = 12;

// BN: rows of x that a tile has room for; a call may use fewer (a multiple of 16).
template <int BN>
struct TilesOf {
    static constexpr int UNIT = BN * 128, STAGE = 2 * UNIT, STAGES = BN > 128 ? 3 : BN == 128 ? 4 : 6;   // of x, two units each
    static constexpr int BUFS = BN > 128 ? 1 : 2;                                   // accumulators
    static constexpr int A_STAGES = 4, A_COLS = kUnitCols / 2;                       // of turned codes, two units each, behind these
    static constexpr int HALF = BN / 2;    // columns of a folding thread
    static constexpr int OUT_COLS = 8;     // that leave at once
    static constexpr int CODE_RING = (BN == 256 ? 24 : BN > 128 ? 48 : BN == 128 ? 64 : 96) * 1024, OUT_BYTES = 8 * OUT_COLS * 32 * 4;
    static constexpr int SMEM = STAGES * STAGE + CODE_RING + OUT_BYTES + 1024 + 768;
    // registers a thread: 96 at launch, dealt out anew by role (warps 0-3, two warpgroups that turn, two that fold)
    static constexpr int FOLD_REGS = BN > 128 ? 160 : 96, TURN_REGS = BN > 128 ? 56 : 96, LEAD_REGS = BN > 128 ? 48 : 96;
    static_assert(2 * FOLD_REGS + 2 * TURN_REGS + LEAD_REGS <= 5 * 96, "as many as the block was launched with");
    static_assert(BUFS * BN + A_STAGES * 2 * A_COLS <= 512, "tensor memory");
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
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
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
    unsigned long long t0 = 0;
    for (int n = 1;; ++n) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((n & 31) != 0) continue;
        if (*abort) return false;
        const unsigned long long now = globaltimer_ns();
        if (t0 == 0) t0 = now;
        else if (now - t0 > kWaitLimitNs) return false;
    }
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

// A lane's results leave: of output o, for `left` rows of x from m0 on.  Registers have no index, so eight rows at a time
// pass through shared memory, in a loop: written out for all of them its instructions came from afar once a tile, and a
// tile took 100000 cycles to leave.
template <typename F>
__device__ __forceinline__ void leave(const LinearArgs &a, const float (&acc)[F::HALF], float *mine, int64_t m0, int left, int64_t o) {
    constexpr int N = F::OUT_COLS;
    const bool on = o < a.g.q;
    const float bias = on && a.bias ? to_f32(a.bias, a.bias_dtype, o) : 0.0f;
    const uint16_t *res = a.residual && on ? static_cast<const uint16_t *>(a.residual) + m0 * a.ldr + o : nullptr;
    uint16_t *y = static_cast<uint16_t *>(a.y) + m0 * a.ldy + o;
#pragma unroll 1
    for (int part = 0; part < F::HALF / N && part * N < left; ++part) {
        const int here = left - part * N;
        uint16_t r[N];                                    // of the residual, on its way
#pragma unroll
        for (int i = 0; i < N; ++i) {
            r[i] = 0;
            if (res && i < here) r[i] = res[i * a.ldr];
        }
#pragma unroll
        for (int q = 0; q < F::HALF / N; ++q)
            if (q == part)
#pragma unroll
                for (int i = 0; i < N; ++i) mine[i * 32] = acc[q * N + i];
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = mine[i * 32] + bias;
        with_activation(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activated<act.value>(v[i]);
        });
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (res) v[i] += a.half ? __half2float(__ushort_as_half(r[i])) : __uint_as_float(static_cast<uint32_t>(r[i]) << 16);
            const uint16_t h = a.half ? __half_as_ushort(__float2half_rn(v[i])) : __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
            if (on && i < here) y[i * a.ldy] = h;
        }
        if (res) res += N * a.ldr;
        y += N * a.ldy;
    }
}

// SHARED: a cluster's CTAs share a tile's columns.
template <int B, int BN, bool HALF, bool SHARED>
__global__ void __launch_bounds__(kTileThreads, 1) k_linear_tiles(const LinearArgs a, const int bn, const __grid_constant__ CUtensorMap xmap,
                                                                  const __grid_constant__ CUtensorMap cmap) {
    using F = TilesOf<BN>;
    using TU = Turn<B, HALF>;
    constexpr int CODES = 8 * 128 * B;                    // bytes of a unit's codes, of 128 outputs
    // Each group of turning warps has a ring of its own: a barrier's phases are told apart by one bit, so whoever waits on it
    // has to see them all.
    constexpr int CODE_FIT = F::CODE_RING / (2 * CODES), CODE_STAGES = CODE_FIT < 12 ? CODE_FIT : 12;
    extern __shared__ uint8_t raw_smem[];
    uint8_t *smem = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);
    uint8_t *code_ring = smem + F::STAGES * F::STAGE;
    float *out_stage = reinterpret_cast<float *>(code_ring + F::CODE_RING);
    uint64_t *x_full = reinterpret_cast<uint64_t *>(code_ring + F::CODE_RING + F::OUT_BYTES), *x_empty = x_full + F::STAGES;
    uint64_t *a_full = x_empty + F::STAGES, *a_empty = a_full + F::A_STAGES;
    uint64_t *code_full = a_empty + F::A_STAGES, *code_empty = code_full + 2 * CODE_STAGES;
    uint64_t *acc_full = code_empty + 2 * CODE_STAGES, *acc_empty = acc_full + 2, *drain = acc_empty + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    static_assert((2 * F::STAGES + 2 * F::A_STAGES + 5 + 4 * CODE_STAGES) * 8 + 8 <= 768, "room for the barriers");
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = SHARED ? static_cast<int>(cluster.block_rank()) : 0, ranks = SHARED ? static_cast<int>(cluster.num_blocks()) : 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // a tile's outputs run fastest; a cluster takes one tile, a CTA by itself every gridDim.x-th
    const int out_tiles = (a.g.row_tiles + 7) / 8;
    const int tiles = out_tiles * static_cast<int>((a.rows + bn - 1) / bn);
    const int first_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(ranks)), tile_step = static_cast<int>(gridDim.x / static_cast<unsigned>(ranks));
    const int begin = static_cast<int>(static_cast<int64_t>(a.g.units) * rank / ranks),
              end = static_cast<int>(static_cast<int64_t>(a.g.units) * (rank + 1) / ranks);
    const int steps = end - begin, stages = (steps + 1) / 2;    // of a tile: units, and pairs of them (the last may lack one)
    // A segment is what a group, or kSegmentUnits of it, has left (one grid a row: the row is the group).
    const int first_group_end = (begin / a.g.group_units + 1) * a.g.group_units;
    auto segment_end = [&](int u, int group_end) { return min(min(u + kSegmentUnits, group_end), end); };
    // groups with one accumulator: a tile's two halves of rows take turns, one's products running while the other is folded
    const int parts = F::BUFS == 1 && a.g.groups > 1 ? 2 : 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::STAGES; ++s) {
            mbar_init(&x_full[s], 1);
            mbar_init(&x_empty[s], 1);
        }
        for (int s = 0; s < F::A_STAGES; ++s) {
            mbar_init(&a_full[s], 4);
            mbar_init(&a_empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], parts == 2 ? 4 : 8);
        }
        for (int s = 0; s < 2 * CODE_STAGES; ++s) {
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
        if constexpr (SHARED) cluster.sync();
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
                const int m0 = tile / out_tiles * bn;
                for (int u = begin; u < end; u += 2, ++n) {
                    ok = wait_on(&x_empty[at.s], at.phase ^ 1u, abort_flag);
                    if (!ok) break;
                    uint8_t *to = smem + at.s * F::STAGE;
                    mbar_arrive_expect_tx(&x_full[at.s], (u + 1 < end ? 2 : 1) * bn * 128);
                    tma_load_2d(&xmap, to, &x_full[at.s], u * kUnitCols, m0);
                    if (u + 1 < end) tma_load_2d(&xmap, to + F::UNIT, &x_full[at.s], (u + 1) * kUnitCols, m0);
                    at.next();
                }
            }
            if (!ok) give_up();
            // the last copy into each stage has landed before the CTA goes on
            for (int64_t k = n > F::STAGES ? n - F::STAGES : 0; k < n; ++k)
                mbar_wait_bounded(&x_full[k % F::STAGES], static_cast<uint32_t>(k / F::STAGES) & 1u, nullptr);
        }
    } else if (warp == 1) {
        const uint32_t idesc = HALF ? idesc_f16_f32(kTileOut, bn / parts) : idesc_bf16_f32(kTileOut, bn / parts);
        const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0), x_empty0 = smem_u32(x_empty), a_empty0 = smem_u32(a_empty), acc0 = smem_u32(acc_full);
        const uint64_t x0 = smem_desc_k128(smem_u32(smem));
        Turnstile<F::STAGES> xs;
        Turnstile<F::A_STAGES> as;
        Turnstile<F::BUFS> acc[2];                        // of either part
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            int seg_end[2] = {begin, begin}, group_end[2] = {first_group_end, first_group_end};
            for (int u = begin; ok && u < end; u += 2) {
                ok = wait_warp_on(&x_full[xs.s], xs.phase, abort_flag) && wait_warp_on(&a_full[as.s], as.phase, abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    if (part == parts) break;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if (u + k == end) break;
                        uint32_t add = 1u;
                        if (u + k == seg_end[part]) {     // a segment begins: its accumulator has been folded
                            ok = ok && wait_warp_on(&acc_empty[part + acc[part].s], acc[part].phase ^ 1u, abort_flag);
                            tc_fence_after();
                            if (u + k == group_end[part]) group_end[part] += a.g.group_units;
                            seg_end[part] = segment_end(u + k, group_end[part]);
                            add = 0u;
                        }
                        if (!ok) break;
                        const uint32_t dst = t0 + static_cast<uint32_t>(part * F::HALF + acc[part].s * BN);
                        const uint64_t db = x0 + static_cast<uint64_t>((xs.s * F::STAGE + k * F::UNIT + part * (bn / 2) * 128) / 16);
                        const uint32_t da = t0 + static_cast<uint32_t>(F::BUFS * BN + (2 * as.s + k) * F::A_COLS);
                        mma_ts_one(dst, da, db, idesc, add);
#pragma unroll
                        for (int q = 1; q < kUnitCols / 16; ++q) mma_ts_one(dst, da + 8u * q, db + 2u * q, idesc, 1u);
                        if (u + k + 1 == seg_end[part]) {
                            commit_one(acc0 + 8u * (part + acc[part].s));
                            acc[part].next();
                        }
                    }
                }
                if (!ok) break;
                commit_one(x_empty0 + 8u * xs.s);
                commit_one(a_empty0 + 8u * as.s);
                xs.next();
                as.next();
            }
        }
        if (!ok && lane == 0) give_up();
        __syncwarp();
        commit_one(smem_u32(drain));                      // nothing is in flight when tensor memory is freed
        mbar_wait_bounded(drain, 0u, nullptr);
    } else if (warp == 2) {
        if (lane == 0) {                                  // (row tiles past the last are zeros)
            Turnstile<CODE_STAGES> at[2];                 // of either group
            int64_t sent[2] = {0, 0};
            int n = 0;                                    // stages so far
            bool ok = true;
            for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
                const int row0 = tile % out_tiles * (kTileOut / kTileRows);
                for (int u = begin; ok && u < end; u += 2, ++n) {
                    const int group = n & 1;
                    Turnstile<CODE_STAGES> &to = at[group];
                    for (int k = 0; k < 2 && u + k < end; ++k) {
                        const int place = group * CODE_STAGES + to.s;
                        ok = wait_on(&code_empty[place], to.phase ^ 1u, abort_flag);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&code_full[place], CODES);
                        tma_load_2d(&cmap, code_ring + place * CODES, &code_full[place], (u + k) * 32 * B, row0);
                        to.next();
                        ++sent[group];
                    }
                }
            }
            if (!ok) give_up();
            for (int group = 0; group < 2; ++group)
                for (int64_t k = sent[group] > CODE_STAGES ? sent[group] - CODE_STAGES : 0; k < sent[group]; ++k)
                    mbar_wait_bounded(&code_full[group * CODE_STAGES + k % CODE_STAGES], static_cast<uint32_t>(k / CODE_STAGES) & 1u, nullptr);
        }
    } else if (warp >= kTurnWarp && warp < kFoldWarp) {
        if constexpr (F::TURN_REGS < 96) fewer_registers<F::TURN_REGS>();
        const int r = lane >> 2, quad = warp & 3, odd = (warp - kTurnWarp) >> 2;
        const uint32_t to = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(F::BUFS * BN);
        uint32_t zero[2][2][TU::LEVELS], w[2][B], v[2][2][4];
        Turnstile<CODE_STAGES> cs;                        // of the next unit's codes
        Turnstile<F::A_STAGES> as;
        bool ok = true;
        auto codes = [&]() {                              // a unit's, into registers
            const int place = odd * CODE_STAGES + cs.s;
            ok = wait_warp_on(&code_full[place], cs.phase, abort_flag);
            if (!ok) return;
#pragma unroll
            for (int i = 0; i < 2; ++i) read_unit<B>(code_ring + place * CODES + (2 * quad + i) * (128 * B), lane, w[i]);
        };
        // Their place in the ring is free once they have been turned, not once they have been asked for: TMA's writes are not
        // held up by loads that are still on their way.
        auto codes_done = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&code_empty[odd * CODE_STAGES + cs.s]);
            cs.next();
        };
        int n = 0;                                        // stages so far: this group has those with n mod 2 == odd
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            const uint32_t *zeros = zero_words(a.g, min(tile % out_tiles * (kTileOut / kTileRows) + 2 * quad, a.g.row_tiles - 1), r);
            // the zeros of this group's next stage, on their way
            uint32_t ahead[2];
            auto load_zeros = [&](int u) {
#pragma unroll
                for (int k = 0; k < 2; ++k) ahead[k] = zeros[a.g.groups > 1 ? static_cast<unsigned>(min(u + k, end - 1)) / static_cast<unsigned>(a.g.group_units) * 8 : 0];
            };
            load_zeros(begin + ((n & 1) != odd ? 2 : 0));
            bool fresh = true;                            // (with one grid a row the first will do for all)
            for (int j = 0; ok && j < stages; ++j, ++n, as.next()) {
                const int u0 = begin + 2 * j, both = u0 + 1 < end ? 2 : 1;
                if ((n & 1) != odd) continue;
                const uint32_t dst = to + static_cast<uint32_t>(2 * as.s * F::A_COLS);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == both) break;
                    if (fresh || a.g.groups > 1) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) TU::zero(zero_of(ahead[k], 2 * i + h), zero[i][h]);
                        fresh = false;
                    }
                    codes();
                    if (!ok) break;
                    TU::unit(w[0], zero[0], v);
                    if (k == 0) {
                        ok = wait_warp_on(&a_empty[as.s], as.phase ^ 1u, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    tmem_st_unit(dst + k * F::A_COLS, v);
                    TU::unit(w[1], zero[1], v);
                    tmem_st_unit(dst + k * F::A_COLS + (16u << 16), v);
                    codes_done();
                }
                if (!ok) break;
                if (a.g.groups > 1) load_zeros(u0 + 4);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&a_full[as.s]);
            }
        }
        if (!ok && lane == 0) give_up();
    } else if (warp >= kFoldWarp) {
        if constexpr (F::FOLD_REGS > 96) more_registers<F::FOLD_REGS>();
        const int quad = warp & 3, side = (warp - kFoldWarp) >> 2, row = quad * 32 + lane;
        const uint32_t from = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(side * F::HALF);
        Turnstile<F::BUFS> buf;
        const int part = parts == 2 ? side : 0, rows0 = parts == 2 ? side * (bn / 2) : side * F::HALF;   // the accumulator's, and the rows' place
        const int cols = parts == 2 ? bn / 2 : min(bn - rows0, F::HALF);   // rows of x it has (none is left, or less, where bn is small)
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += tile_step) {
            const int out_tile = tile % out_tiles;
            const int64_t row_tile = min(out_tile * (kTileOut / kTileRows) + row / kTileRows, a.g.row_tiles - 1);
            const int64_t m0 = static_cast<int64_t>(tile / out_tiles) * bn + rows0;
            float acc[F::HALF];
#pragma unroll
            for (int i = 0; i < F::HALF; ++i) acc[i] = 0.0f;
            const float *scales = a.g.scales + row_tile * a.g.groups * kTileRows + row % kTileRows;
            int g = a.g.groups > 1 ? begin / a.g.group_units : 0;
            float ahead = scales[g * kTileRows];          // of the next segment
            for (int u = begin, group_end = first_group_end; u < end; buf.next()) {
                const float scale = ahead;
                u = segment_end(u, group_end);
                if (u == group_end) {
                    group_end += a.g.group_units;
                    if (g + 1 < a.g.groups) ahead = scales[++g * kTileRows];
                }
                ok = wait_warp_on(&acc_full[part + buf.s], buf.phase, abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < F::HALF / 16; ++q) {  // (columns past bn hold anything, and stay in theirs)
                    float v[16];
                    tmem_ld_16(from + static_cast<uint32_t>(buf.s * BN + q * 16), v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[q * 16 + i] = fmaf(scale, v[i], acc[q * 16 + i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[part + buf.s]);
            }
            if constexpr (SHARED) {
                // x's ring is free for the sums, [row of x][output], once every product of the tile has been taken: either side
                // has waited for its own part's, so they meet (and where a wait gave up too, lest the other side wait for ever)
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
            if (!ok) break;
            if constexpr (SHARED) {
                float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
                for (int i = 0; i < F::HALF; ++i)
                    if (i < cols) sums[(rows0 + i) * kTileOut + row] = acc[i];
            } else {
                const int64_t o = static_cast<int64_t>(out_tile) * kTileOut + row;
                const int64_t left = min(a.rows - m0, static_cast<int64_t>(cols));   // rows of x that are there
                leave<F>(a, acc, out_stage + (warp - kFoldWarp) * (F::OUT_COLS * 32) + lane, m0, static_cast<int>(left), o);
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
    if constexpr (SHARED) {                               // the cluster's CTAs take rows of x in turn
        const int64_t m0 = static_cast<int64_t>(first_tile / out_tiles) * bn, out0 = static_cast<int64_t>(first_tile % out_tiles) * kTileOut;
        const float *sums = reinterpret_cast<const float *>(smem);
        const int failed = *abort_flag;
        if (!failed)
            with_activation(a.act, [&](auto act) {
                // four outputs of a row a thread, a warp a row
                const int64_t i0 = out0 + 4 * lane;
                float bias[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) bias[k] = a.bias && i0 + k < a.g.q ? to_f32(a.bias, a.bias_dtype, i0 + k) : 0.0f;
                const int here = static_cast<int>(min(a.rows - m0, static_cast<int64_t>(bn)));
#pragma unroll 1
                for (int tok = (warp - kFoldWarp) * ranks + rank; tok < here; tok += 8 * ranks) {
                    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
                    for (int q = 0; q < ranks; ++q) {
                        const float4 x = *reinterpret_cast<const float4 *>(cluster.map_shared_rank(sums, q) + tok * kTileOut + 4 * lane);
                        v[0] += x.x;
                        v[1] += x.y;
                        v[2] += x.z;
                        v[3] += x.w;
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (i0 + k < a.g.q) finish<act.value>(a, v[k], m0 + tok, i0 + k, bias[k]);
                }
            });
    }
    meet();
}

template <int B, int BN, bool HALF, bool SHARED>
cudaError_t launch_tiles_as(const LinearArgs &a, const TilesPlan &plan, cudaStream_t s) {
    using F = TilesOf<BN>;
    CUtensorMap map, codes;
    if (!(HALF ? make_tmap_f16 : make_tmap_bf16)(&map, a.x, static_cast<uint64_t>(a.rows), static_cast<uint64_t>(a.g.p),
                                                 static_cast<uint64_t>(a.ldx), static_cast<uint32_t>(plan.rows)) ||
        !make_tmap_words(&codes, a.g.codes, static_cast<uint64_t>(a.g.row_tiles), static_cast<uint64_t>(a.g.units) * 32 * B, 32 * B, kTileOut / kTileRows))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> raised{0};
    const void *kernel = reinterpret_cast<const void *>(k_linear_tiles<B, BN, HALF, SHARED>);
    cudaError_t e = raise_limit(kernel, F::SMEM, raised);
    if (e != cudaSuccess) return e;
    const int64_t tiles = ceil_div(a.g.q, kTileOut) * ceil_div(a.rows, plan.rows), sms = linear_sms();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(plan.ranks > 1 ? tiles * plan.ranks : tiles < sms ? tiles : sms));
    cfg.blockDim = dim3(kTileThreads);
    cfg.dynamicSmemBytes = F::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(plan.ranks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_linear_tiles<B, BN, HALF, SHARED>, a, plan.rows, map, codes);
}

template <int B, int BN>
cudaError_t launch_tiles_type(const LinearArgs &a, const TilesPlan &plan, cudaStream_t s) {
    if (plan.ranks > 1) return a.half ? launch_tiles_as<B, BN, true, true>(a, plan, s) : launch_tiles_as<B, BN, false, true>(a, plan, s);
    return a.half ? launch_tiles_as<B, BN, true, false>(a, plan, s) : launch_tiles_as<B, BN, false, false>(a, plan, s);
}

template <int B>
cudaError_t launch_tiles_bits(const LinearArgs &a, cudaStream_t s) {
    const TilesPlan plan = tiles_plan(a);
    if (plan.room == 64) return launch_tiles_type<B, 64>(a, plan, s);
    if (plan.room == 128) return launch_tiles_type<B, 128>(a, plan, s);
    return launch_tiles_type<B, B == 8 ? 224 : 256>(a, plan, s);
}

}  // namespace
}  // namespace qe
