// Products with a quantized layer for a few rows of x: y = act(x What^T + bias) + residual.
//
// Bound by reading the codes once, closely followed by turning them into operands: at
// 6.8 TB/s an SM is handed some 47 4-bit codes a cycle.  A warp takes RT row tiles of 16
// outputs and a run of columns, reads their codes as two streams straight into registers,
// a few units ahead, turns each pair of codes with two or three instructions into 16-bit
// floats c - z (exact) and multiplies them with up to 8 NT rows of x on m16n8k16, the outputs
// in the 16-high side.  Products are exact and sums binary32; the scale comes in at the end, or at
// the end of every group.  The warps of a CTA share its outputs' columns out among them, and so
// do the CTAs of a cluster: their sums meet in shared memory, warps and CTAs in order, so that
// results do not depend on who is first.
#pragma once

#include <cooperative_groups.h>

#include "qe_internal.h"
#include "qe_linear.cuh"

namespace qe {
namespace {

constexpr int kRowWarps = 8;

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

template <int B, int RT, int NT>
struct RowsOf {
    static constexpr int ROWS = kTileRows * RT, TOKENS = 8 * NT, LD = ROWS + 4;
    static constexpr int AHEAD = 4 * (RT * B + 8 * NT) <= 64 ? 4 : 3 * (RT * B + 8 * NT) <= 64 ? 3 : 2;   // units in registers
    static constexpr int SMEM = kRowWarps * TOKENS * LD * 4;
};

// Eight columns of a row of x from column k on; columns past p, and rows that are not there, are zeros.
__device__ __forceinline__ uint4 load_x8(const LinearArgs &a, const uint16_t *row, bool on, int64_t k) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (!on || k >= a.g.p) return v;
    if (a.x_vec && k + 8 <= a.g.p) return *reinterpret_cast<const uint4 *>(row + k);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = k + 2 * i < a.g.p ? row[k + 2 * i] : 0u, hi = k + 2 * i + 1 < a.g.p ? row[k + 2 * i + 1] : 0u;
        w[i] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int B, int RT, int NT, bool HALF, bool GROUPED>
__global__ void __launch_bounds__(kRowWarps * 32) k_linear_rows(const LinearArgs a) {
    using F = RowsOf<B, RT, NT>;
    using TU = Turn<B, HALF>;
    constexpr int AHEAD = F::AHEAD;
    extern __shared__ __align__(16) float met[];          // [warp][token][row], then [0]: this CTA's sums
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ranks = static_cast<int>(cluster.num_blocks());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    const int tile0 = static_cast<int>(blockIdx.x / static_cast<unsigned>(ranks)) * RT;
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * F::TOKENS;
    const int64_t units = a.g.units;
    const int shares = ranks * kRowWarps, share = rank * kRowWarps + warp;
    const int begin = static_cast<int>(units * share / shares), end = static_cast<int>(units * (share + 1) / shares);

    int tile[RT];
    const uint8_t *code[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {                        // (tiles that are not there repeat the last one, unused)
        tile[i] = min(tile0 + i, a.g.row_tiles - 1);
        code[i] = a.g.codes + (tile[i] * units + begin) * (128 * B);
    }
    const uint16_t *xr[NT];
    bool on[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t m = m0 + 8 * n + r;
        on[n] = m < a.rows;
        xr[n] = static_cast<const uint16_t *>(a.x) + (on[n] ? m : 0) * a.ldx;
    }

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
    uint32_t w[AHEAD][RT][B];
    uint4 x[AHEAD][NT][2];
    auto fetch = [&](int u, uint32_t (&wd)[RT][B], uint4 (&xd)[NT][2]) {
#pragma unroll
        for (int i = 0; i < RT; ++i) load_unit<B>(code[i] + static_cast<int64_t>(u - begin) * (128 * B), lane, wd[i]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) xd[n][c] = load_x8(a, xr[n], on[n], static_cast<int64_t>(u) * kUnitCols + 32 * c + 8 * t);
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (begin + s < end) fetch(begin + s, w[s], x[s]);

    uint32_t zero[RT][2][TU::LEVELS];
    float scale[RT][2];
    int next_grid = begin;                                // unit at which the grids change
    auto grids = [&](int g) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = (static_cast<int64_t>(tile[i]) * a.g.groups + g) * kTileRows + r + 8 * h;
                scale[i][h] = a.g.scales[at];
                TU::zero(static_cast<float>(a.g.zeros[at]), zero[i][h]);
            }
    };
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
    if constexpr (!GROUPED) grids(0);
    for (int u0 = begin; u0 < end; u0 += AHEAD) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int u = u0 + s;
            if (u >= end) break;
            if constexpr (GROUPED) {
                if (u == next_grid) {
                    if (u > begin) fold();
                    const int g = u / a.g.group_units;
                    grids(g);
                    next_grid = (g + 1) * a.g.group_units;
                }
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                uint32_t v[2][2][4];
                TU::unit(w[s][i], zero[i], v);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        mma_16816<HALF>(sum[i][n], v[c][0][0], v[c][1][0], v[c][0][1], v[c][1][1], x[s][n][c].x, x[s][n][c].y);
                        mma_16816<HALF>(sum[i][n], v[c][0][2], v[c][1][2], v[c][0][3], v[c][1][3], x[s][n][c].z, x[s][n][c].w);
                    }
            }
            if (u + AHEAD < end) fetch(u + AHEAD, w[s], x[s]);
        }
    }
    if constexpr (GROUPED) {
        if (begin < end) fold();
    }

    // ---- the warps' sums meet, then the cluster's ----
    float *mine = met + warp * (F::TOKENS * F::LD);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = GROUPED ? total[GROUPED ? i : 0][GROUPED ? n : 0][e] : sum[i][n][e] * (begin < end ? scale[i][e >> 1] : 0.0f);
                mine[(8 * n + 2 * t + (e & 1)) * F::LD + kTileRows * i + r + 8 * (e >> 1)] = v;
            }
    __syncthreads();
    constexpr int ALL = F::TOKENS * F::ROWS;
    for (int e = threadIdx.x; e < ALL; e += kRowWarps * 32) {
        float *p = met + (e / F::ROWS) * F::LD + e % F::ROWS;
        float v = p[0];
#pragma unroll
        for (int k = 1; k < kRowWarps; ++k) v += p[k * (F::TOKENS * F::LD)];
        p[0] = v;
    }
    if (ranks > 1) cluster.sync();
    else __syncthreads();
    for (int e = rank * (kRowWarps * 32) + threadIdx.x; e < ALL; e += ranks * kRowWarps * 32) {
        const int tok = e / F::ROWS, row = e % F::ROWS;
        const int64_t i = static_cast<int64_t>(tile0) * kTileRows + row, m = m0 + tok;
        if (i >= a.g.q || m >= a.rows) continue;
        float v = 0.0f;
        for (int k = 0; k < ranks; ++k) v += (ranks > 1 ? cluster.map_shared_rank(met, k) : met)[tok * F::LD + row];
        put(a, finished(a, v, m, i, a.bias ? to_f32(a.bias, a.bias_dtype, i) : 0.0f), m, i);
    }
    if (ranks > 1) cluster.sync();                        // nobody leaves while its sums are read
}

template <int B, int RT, int NT, bool HALF, bool GROUPED>
cudaError_t launch_rows_as(const LinearArgs &a, cudaStream_t s) {
    using F = RowsOf<B, RT, NT>;
    const int64_t groups = ceil_div(a.g.row_tiles, RT), blocks = ceil_div(a.rows, F::TOKENS);
    int ranks = 1;
    while (ranks < 8 && groups * blocks * ranks < 304 && a.g.units >= 2 * ranks * kRowWarps * 2) ranks *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(groups * ranks), static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kRowWarps * 32);
    cfg.dynamicSmemBytes = F::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(ranks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    static_assert(F::SMEM <= 48 * 1024, "no limit to raise");
    return cudaLaunchKernelEx(&cfg, k_linear_rows<B, RT, NT, HALF, GROUPED>, a);
}

template <int B, int RT, int NT>
cudaError_t launch_rows_type(const LinearArgs &a, cudaStream_t s) {
    if (a.g.groups > 1) return a.half ? launch_rows_as<B, RT, NT, true, true>(a, s) : launch_rows_as<B, RT, NT, false, true>(a, s);
    return a.half ? launch_rows_as<B, RT, NT, true, false>(a, s) : launch_rows_as<B, RT, NT, false, false>(a, s);
}

template <int B>
cudaError_t launch_rows_bits(const LinearArgs &a, cudaStream_t s) {
    constexpr int RT = B == 8 ? 1 : 2;
    if (a.rows <= 8) return launch_rows_type<B, RT, 1>(a, s);
    if (a.rows <= 16) return launch_rows_type<B, RT, 2>(a, s);
    return launch_rows_type<B, RT, 4>(a, s);
}

}  // namespace
}  // namespace qe
