// Products with a quantized layer for a few rows of x: y = act(x What^T + bias) + residual.
//
// Bound by reading the codes once, closely followed by turning them into operands: at
// 6.8 TB/s an SM is handed some 47 4-bit codes a cycle, and the integer pipe takes two cycles
// for a warp's instruction.  A warp takes RT row tiles of 16 outputs, reads their codes as
// streams straight into registers, two to four units of 64 columns ahead, turns each pair of codes
// with two or three instructions into 16-bit floats c - z (exact) and multiplies them with up
// to 8 NT rows of x on m16n8k16, the outputs in the 16-high side.  Products are exact and sums
// binary32; the scale comes in at the end, or at the end of every group.  Accumulators are emptied
// every kSegmentUnits units (LONG): of groups that are longer into registers; with one grid a row, where
// a CTA has more than twice as many units, into shared memory, a place of the thread's own for each.
// (In one kernel for all calls it took 100 us instead of 97 for the first size below, and 319 instead
// of 291 for it in groups of 128 at 8 bits.)  The eight warps of a CTA share x, which passes through
// shared memory 256 columns at a time (swizzled by 16 bytes, read by ldmatrix).  The CTAs of a cluster
// share a layer's columns out among them: their sums meet in shared memory, in order, so that results
// do not depend on who is first.
//
// Measured (us, caches out of L2; of codes read): 5 x 14848 x 59392, fp16, 4 bits 94 (4.7 TB/s), 3 bits 98 (3.4 TB/s: a unit's turning
// is the same work for fewer bytes; the integer pipe is busy 66% of the time, issue slots 58%), 8 bits 162 (5.4 TB/s), bf16 104, 104
// and 229 (five instructions for two 8-bit codes); 1 x 4096 x 11008, 4 bits 14, 1 x 4096 x 4096, 3 bits 10 to 13 (the launch, a cluster's
// meeting and the first loads' way take most of it); 24 x 11008 x 4096, 4 bits in groups of 128 19 to 22.
#pragma once

#include <cooperative_groups.h>

#include "qe_internal.h"
#include "qe_linear.cuh"

namespace qe {
namespace {

constexpr int kRowWarps = 8, kChunk = 4;   // kChunk: units of x in a stage
constexpr int kSegmentChunks = kSegmentUnits / kChunk;

template <bool HALF>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int OFFSET>
__device__ __forceinline__ void ldmatrix_x4(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4 + %5];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at), "n"(OFFSET));
}

// f(0) .. f(N - 1), as constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

// Units of codes on their way in a warp's registers.
__host__ __device__ constexpr int rows_ahead(int B, int RT) { return RT == 2 ? 2 : B == 8 ? 2 : 4; }

template <int RT, int NT>
struct RowsOf {
    static constexpr int ROWS = kRowWarps * kTileRows * RT, TOKENS = 8 * NT, LD = ROWS + 4;
    static constexpr int UNIT_BYTES = TOKENS * 128, STAGE = kChunk * UNIT_BYTES, STAGES = 3;
    static constexpr int SUMS = TOKENS * LD * 4;
    static constexpr int SMEM = STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS;
    static constexpr int KEPT = RT * NT * 4 * kRowWarps * 32 * 4;           // sums of earlier segments
    static constexpr int PIECES = TOKENS * 8 * kChunk / (kRowWarps * 32);   // 16-byte pieces of a stage a thread brings
};

// `bytes` (0 .. 16) from global memory, the rest zeros.
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes) : "memory");
}

// CTAs that an SM holds, by registers.
__host__ __device__ constexpr int rows_ctas(int NT) { return NT == 1 ? 3 : 2; }

template <int B, int RT, int NT, bool HALF, bool GROUPED, bool LONG>
__global__ void __launch_bounds__(kRowWarps * 32, rows_ctas(NT)) k_linear_rows(const LinearArgs a) {
    using F = RowsOf<RT, NT>;
    using TU = Turn<B, HALF>;
    extern __shared__ __align__(128) uint8_t smem[];
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    const int tile0 = static_cast<int>(blockIdx.x / static_cast<unsigned>(ranks)) * (kRowWarps * RT);
    // (of calls that are made, 0; without the grid's second axis the main loop is compiled to something up to 11% slower:
    // 30 x 14848 x 14848, 4 bits, fp16 57 / 63 us)
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * F::TOKENS;
    const int units = a.g.units;
    const int begin = static_cast<int>(static_cast<int64_t>(units) * rank / ranks), end = static_cast<int>(static_cast<int64_t>(units) * (rank + 1) / ranks);
    const int chunks = (end - begin + kChunk - 1) / kChunk;

    int tile[RT];
    const uint8_t *code[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {                        // (tiles that are not there repeat the last one, unused)
        tile[i] = min(tile0 + warp * RT + i, a.g.row_tiles - 1);
        code[i] = a.g.codes + (static_cast<int64_t>(tile[i]) * units + begin) * (128 * B);
    }
    constexpr int AHEAD = rows_ahead(B, RT);
    uint32_t w[AHEAD][RT][B];
    auto fetch = [&](int s) {                             // unit s behind the beginning of the chunk that `code` stands at
#pragma unroll
        for (int i = 0; i < RT; ++i) load_unit<B>(code[i] + s * (128 * B), w[s % AHEAD][i]);
    };
#pragma unroll
    for (int i = 0; i < RT; ++i) code[i] += B == 3 ? 4 * lane : B == 2 ? 8 * lane : 16 * lane;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (begin + s < end) fetch(s);

    // x: piece e of a stage is row e / 32's 16 bytes e mod 32: a thread brings the same piece of every eighth row
    const uint32_t ring = smem_u32(smem);
    const int pc = threadIdx.x & 31, row0 = threadIdx.x >> 5;
    const uint32_t x_to = ring + (pc >> 3) * F::UNIT_BYTES + row0 * 128 + (((pc & 7) ^ (row0 & 7)) << 4);
    const int64_t x_col = static_cast<int64_t>(begin) * kUnitCols + 8 * pc, x_step = 8 * a.ldx;
    const uint16_t *x_from = static_cast<const uint16_t *>(a.x) + (m0 + row0) * a.ldx + x_col;
    const int x_rows = a.rows - m0 - row0 <= 0 ? 0 : static_cast<int>((a.rows - m0 - row0 + 7) / 8);   // of the thread's, that are there
    const int x_chunks = a.x_vec ? static_cast<int>((a.g.p - static_cast<int64_t>(begin) * kUnitCols) / (kChunk * kUnitCols)) : 0;   // whole ones
    auto bring = [&](int c) {
        if (c < chunks) {
            const uint32_t dst = x_to + (c % F::STAGES) * F::STAGE;
            const uint16_t *src = x_from + static_cast<int64_t>(c) * (kChunk * kUnitCols);
            if (c < x_chunks) {
#pragma unroll
                for (int j = 0; j < F::PIECES; ++j)
                    cp_async16_part(dst + j * 1024, j < x_rows ? src + j * x_step : static_cast<const uint16_t *>(a.x), j < x_rows ? 16 : 0);
            } else {                                      // the end of a row, or rows that are not aligned
                const int64_t left = a.g.p - x_col - static_cast<int64_t>(c) * (kChunk * kUnitCols);
#pragma unroll 1
                for (int j = 0; j < F::PIECES; ++j) {
                    const int n = j >= x_rows || left <= 0 ? 0 : left >= 8 ? 8 : static_cast<int>(left);
                    uint32_t v[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        v[q] = (2 * q < n ? src[j * x_step + 2 * q] : 0u) | (2 * q + 1 < n ? static_cast<uint32_t>(src[j * x_step + 2 * q + 1]) << 16 : 0u);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + j * 1024), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int c = 0; c < F::STAGES - 1; ++c) bring(c);

    float sum[RT][NT][4], total[GROUPED ? RT : 1][GROUPED ? NT : 1][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[i][n][e] = 0.0f;
                if constexpr (GROUPED) total[i][n][e] = 0.0f;
            }
    uint32_t zero[RT][2][TU::LEVELS];
    float scale[RT][2];
    int next_grid = begin, group = GROUPED ? begin / a.g.group_units : 0;   // unit at which the grids change, and to which
    float scale_ahead[RT][2];                             // the next group's
    uint32_t zero_ahead[RT];
    const float *scales[RT];
    const uint32_t *zeros[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        scales[i] = a.g.scales + static_cast<int64_t>(tile[i]) * a.g.groups * kTileRows + r;
        zeros[i] = zero_words(a.g, tile[i], r);
    }
    auto load_grids = [&](int g) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) scale_ahead[i][h] = scales[i][g * kTileRows + 8 * h];
            zero_ahead[i] = zeros[i][g * 8];
        }
    };
    auto turn_grids = [&]() {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                scale[i][h] = scale_ahead[i][h];
                TU::zero(zero_of(zero_ahead[i], 2 * (tile[i] & 1) + h), zero[i][h]);
            }
    };
    load_grids(group);
    auto fold = [&]() {
        if constexpr (GROUPED) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        total[i][n][e] = fmaf(scale[i][e >> 1], sum[i][n][e], total[i][n][e]);
                        sum[i][n][e] = 0.0f;
                    }
        }
    };
    if constexpr (!GROUPED) turn_grids();
    float *kept = reinterpret_cast<float *>(smem + F::SMEM) + threadIdx.x;   // one grid a row: sums of the segments before
    auto keep = [&](bool first) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float *place = kept + ((i * NT + n) * 4 + e) * (kRowWarps * 32);
                    *place = first ? sum[i][n][e] : *place + sum[i][n][e];
                    sum[i][n][e] = 0.0f;
                }
    };
    // matrix j of an ldmatrix: rows' piece 4 c + j; lane 8 j + i addresses row i
    const int mrow = lane & 7, mpiece = lane >> 3;
    const uint32_t mat0 = ring + mrow * 128 + ((mpiece ^ mrow) << 4), mat1 = ring + mrow * 128 + (((4 + mpiece) ^ mrow) << 4);
    auto chunk = [&](int c) {
        asm volatile("cp.async.wait_group %0;" ::"n"(F::STAGES - 2) : "memory");
        __syncthreads();                                  // the chunk is there, and everyone has done with the one before
        bring(c + F::STAGES - 1);
        const uint32_t stage = (c % F::STAGES) * F::STAGE, at0 = mat0 + stage, at1 = mat1 + stage;
        const int u0 = begin + c * kChunk;
        auto unit = [&](auto s, bool more) {
            if constexpr (GROUPED) {
                if (u0 + s.value == next_grid) {
                    if (u0 + s.value > begin) fold();
                    turn_grids();
                    if (++group < a.g.groups) load_grids(group);
                    next_grid = group * a.g.group_units;
                }
            }
            // the few registers of x first, where there are more row tiles; else the turned codes
            uint32_t x[NT][2][4], v[2][2][4];
            auto operand = [&](auto n) {
                ldmatrix_x4<s.value * F::UNIT_BYTES + n.value * 1024>(at0, x[n.value][0]);
                ldmatrix_x4<s.value * F::UNIT_BYTES + n.value * 1024>(at1, x[n.value][1]);
            };
            auto products = [&](int i, int n) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    mma_16816<HALF>(sum[i][n], v[q][0][0], v[q][1][0], v[q][0][1], v[q][1][1], x[n][q][0], x[n][q][1]);
                    mma_16816<HALF>(sum[i][n], v[q][0][2], v[q][1][2], v[q][0][3], v[q][1][3], x[n][q][2], x[n][q][3]);
                }
            };
            if constexpr (RT > 1) each<NT>(operand);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                TU::unit(w[s.value % AHEAD][i], zero[i], v);
                if (i + 1 == RT && more) fetch(s.value + AHEAD);
                each<NT>([&](auto n) {
                    if constexpr (RT == 1) operand(n);
                    products(i, n.value);
                });
            }
        };
        if (u0 + kChunk + AHEAD <= end) each<kChunk>([&](auto s) { unit(s, true); });
        else
            each<kChunk>([&](auto s) {
                if (u0 + s.value < end) unit(s, u0 + s.value + AHEAD < end);
            });
#pragma unroll
        for (int i = 0; i < RT; ++i) code[i] += kChunk * 128 * B;
    };
    if constexpr (LONG) {
        for (int c = 0; c < chunks;) {
            for (const int stop = min(chunks, c + kSegmentChunks); c < stop; ++c) chunk(c);
            if constexpr (GROUPED) fold();
            else keep(c <= kSegmentChunks);
        }
    } else {
        for (int c = 0; c < chunks; ++c) chunk(c);
        if constexpr (GROUPED) {
            if (begin < end) fold();
        }
    }

    // ---- the cluster's sums meet ----
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float *met = reinterpret_cast<float *>(smem);         // [row of x][output]
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float all = LONG && !GROUPED ? kept[((i * NT + n) * 4 + e) * (kRowWarps * 32)] : sum[i][n][e];
                const float v = GROUPED ? total[GROUPED ? i : 0][GROUPED ? n : 0][e] : begin < end ? all * scale[i][e >> 1] : 0.0f;
                met[(8 * n + 2 * t + (e & 1)) * F::LD + kTileRows * (warp * RT + i) + r + 8 * (e >> 1)] = v;
            }
    if (ranks > 1) cluster.sync();
    else __syncthreads();
    constexpr int ALL = F::TOKENS * F::ROWS;
    const int here = a.rows - m0 < F::TOKENS ? static_cast<int>(a.rows - m0) * F::ROWS : ALL;
    with_activation(a.act, [&](auto act) {
        for (int e = rank * (kRowWarps * 32) + threadIdx.x; e < here; e += ranks * kRowWarps * 32) {
            const int tok = e / F::ROWS, row = e % F::ROWS;
            const int64_t i = static_cast<int64_t>(tile0) * kTileRows + row;
            if (i >= a.g.q) continue;
            float v = 0.0f, of[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) of[k] = k < ranks ? (ranks > 1 ? cluster.map_shared_rank(met, k) : met)[tok * F::LD + row] : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) v += of[k];       // in order
            finish<act.value>(a, v, m0 + tok, i, a.bias ? to_f32(a.bias, a.bias_dtype, i) : 0.0f);
        }
    });
    if (ranks > 1) cluster.sync();                        // nobody leaves while its sums are read
}

template <int B, int RT, int NT, bool HALF, bool GROUPED, bool LONG>
cudaError_t launch_rows_as(const LinearArgs &a, int ranks, cudaStream_t s) {
    using F = RowsOf<RT, NT>;
    const int64_t groups = ceil_div(a.g.row_tiles, RT * kRowWarps), blocks = ceil_div(a.rows, F::TOKENS);
    constexpr int smem = F::SMEM + (LONG && !GROUPED ? F::KEPT : 0);
    static std::atomic<uint64_t> raised{0};
    const void *kernel = reinterpret_cast<const void *>(k_linear_rows<B, RT, NT, HALF, GROUPED, LONG>);
    if (smem > 48 * 1024) {
        const cudaError_t e = raise_limit(kernel, smem, raised);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(groups * ranks), static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kRowWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(ranks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_linear_rows<B, RT, NT, HALF, GROUPED, LONG>, a);
}

template <int B, int RT, int NT>
cudaError_t launch_rows_type(const LinearArgs &a, int ranks, cudaStream_t s) {
    if (a.g.groups > 1) {
        if (a.g.group_units > kSegmentUnits)
            return a.half ? launch_rows_as<B, RT, NT, true, true, true>(a, ranks, s) : launch_rows_as<B, RT, NT, false, true, true>(a, ranks, s);
        return a.half ? launch_rows_as<B, RT, NT, true, true, false>(a, ranks, s) : launch_rows_as<B, RT, NT, false, true, false>(a, ranks, s);
    }
    if (ceil_div(a.g.units, ranks) > 2 * kSegmentUnits)
        return a.half ? launch_rows_as<B, RT, NT, true, false, true>(a, ranks, s) : launch_rows_as<B, RT, NT, false, false, true>(a, ranks, s);
    return a.half ? launch_rows_as<B, RT, NT, true, false, false>(a, ranks, s) : launch_rows_as<B, RT, NT, false, false, false>(a, ranks, s);
}

template <int B, int RT>
cudaError_t launch_rows_tokens(const LinearArgs &a, int ranks, cudaStream_t s) {
    if (a.rows <= 8) return launch_rows_type<B, RT, 1>(a, ranks, s);
    if constexpr (RT == 1) {
        if (a.rows <= 16) return launch_rows_type<B, 1, 2>(a, ranks, s);
        return a.rows <= 24 ? launch_rows_type<B, 1, 3>(a, ranks, s) : launch_rows_type<B, 1, 4>(a, ranks, s);
    }
    return cudaErrorInvalidValue;
}

template <int B>
cudaError_t launch_rows_bits(const LinearArgs &a, cudaStream_t s) {
    const RowsPlan plan = rows_plan(a);
    if constexpr (B != 8) {
        if (plan.tiles == 2) return launch_rows_tokens<B, 2>(a, plan.ranks, s);
    }
    return launch_rows_tokens<B, 1>(a, plan.ranks, s);
}

}  // namespace
}  // namespace qe
