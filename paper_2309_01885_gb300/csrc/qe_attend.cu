// Attention over the 4-bit key/value cache, few query rows per kv head (single
// tokens, a few drafted ones): out_i = sum_j softmax_j(scale q_i . k^_j) v^_j.
//
// Bound by reading the cache once (D + 8 D / G bytes per token and kv head for
// keys and values together), closely followed by the instructions that turn
// codes into matrix operands: at 6.8 TB/s an SM is handed some 40 codes a cycle
// and issues 128 lanes' instructions.  So the query rows that share a kv head
// sit together in the 8-wide side of m16n8k16, each code is unpacked once for
// all of them, and the unpacking is kept to a minimum:
//   keys   scores are taken transposed, S^T[token][row] = K Q^T.  Masking a code
//          word with 0x000f000f << 4 p leaves pairs of fp16 subnormals c 2^-24 or
//          c 2^-20, which the tensor core multiplies exactly; the power of two
//          goes into Q's fragment, the zero point enters as the accumulator's
//          start -z sum(q), the scale once per group and token in fp32.  Q rows
//          are scaled by a power of two into fp16's range (exact but for values
//          2^-39 below the row's largest).
//   values O^T[channel][row] = V^T P^T.  c - z is exact in bf16 and times the bf16
//          scale rounds once, as a cache held in bf16 would; P is rounded to bf16
//          too (2^-9 relative, a tenth of the 4-bit step and averaged over tokens),
//          sums and softmax statistics stay in fp32.
// The 16 x 8 score fragment becomes P^T's fragment by an 8 x 8 transpose in the
// warp.  A warp walks 16-token steps on its own, fed by bulk copies into a ring
// of its own, and keeps its own running maximum, which it raises only when a
// score exceeds it by 2^8 (P stays below 2^8, no rounding suffers); warps meet in
// shared memory at the end, pieces of a long sequence in a second kernel.
#include <cuda_fp16.h>
#include <math_constants.h>

#include "qe_attend.h"
#include "qe_internal.h"

namespace qe {
namespace {

constexpr int kWarps = 4;
constexpr float kRaise = 8.0f;            // log2 of how far a score may exceed the running maximum
constexpr float kFloor = -1.0e30f;        // the running maximum before the first visible score

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}

template <int N>
__device__ __forceinline__ void lds_words(const uint8_t *p, uint32_t (&w)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 t = reinterpret_cast<const uint4 *>(p)[i];
            w[4 * i] = t.x; w[4 * i + 1] = t.y; w[4 * i + 2] = t.z; w[4 * i + 3] = t.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint2 t = reinterpret_cast<const uint2 *>(p)[i];
            w[2 * i] = t.x; w[2 * i + 1] = t.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    }
}

// One query row's eight channels from `at`, as floats; channels past `dim` are zero.
__device__ __forceinline__ void load_q8(const AttendArgs &a, int64_t row, int head, int at, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    if (at >= a.g.dim) return;            // dim is a multiple of 8
    const int64_t off = row * a.q_row + head * a.q_head + at;
    if (a.half) {
        const __half *p = reinterpret_cast<const __half *>(a.Q) + off;
        if (a.q_vec) {
            union { uint4 u; __half e[8]; } t;
            t.u = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __half2float(t.e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __half2float(p[i]);
        }
    } else {
        const __nv_bfloat16 *p = reinterpret_cast<const __nv_bfloat16 *>(a.Q) + off;
        if (a.q_vec) {
            union { uint4 u; __nv_bfloat16 e[8]; } t;
            t.u = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __bfloat162float(t.e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __bfloat162float(p[i]);
        }
    }
}

__device__ __forceinline__ void store_out(const AttendArgs &a, int64_t row, int head, int d, float v) {
    const int64_t off = row * a.o_row + head * a.o_head + d;
    if (a.half) reinterpret_cast<__half *>(a.out)[off] = __float2half_rn(v);
    else reinterpret_cast<__nv_bfloat16 *>(a.out)[off] = __float2bfloat16_rn(v);
}

// Four channels of a finished row, from the unnormalised sums relative to the maximum `m` (log2 units).
__device__ __forceinline__ void finish(const AttendArgs &a, int64_t row, int head, int d, const float4 &v, float m, float l) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;       // a row that sees nothing is zero; NaN stays
    store_out(a, row, head, d, v.x * inv);
    store_out(a, row, head, d + 1, v.y * inv);
    store_out(a, row, head, d + 2, v.z * inv);
    store_out(a, row, head, d + 3, v.w * inv);
    if (d == 0 && a.lse)
        a.lse[row * a.q_heads + head] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * 0.693147180559945309f;
}

// C chunks of 32 channels, GC chunks to a group, NT tiles of 8 query rows.
template <int C, int GC, int NT>
struct RowsCfg {
    static constexpr int D = 32 * C, NG = C / GC, ROWS = 8 * NT;
    static constexpr int CODE_BYTES = 8 * D;              // 16 tokens' key (or value) codes
    static constexpr int GRID_BYTES = 64 * NG;
    static constexpr int STEP_BYTES = 2 * CODE_BYTES + 2 * GRID_BYTES;
    static constexpr int STAGES = 4;
    static constexpr int RING = STAGES * STEP_BYTES;      // one warp's
    static constexpr int JOIN = ROWS * (D + 4) * 4 + 2 * ROWS * 4;   // one warp's O, m and l at the end
    static constexpr int WARP_BYTES = RING > JOIN ? RING : JOIN;
    static constexpr int SMEM = kWarps * WARP_BYTES + kWarps * STAGES * 8;
};

template <int C, int GC, int NT>
__global__ void __launch_bounds__(kWarps * 32) k_attend_rows(const AttendArgs a) {
    using F = RowsCfg<C, GC, NT>;
    constexpr int D = F::D, NG = F::NG, STAGES = F::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, t = lane & 3;
    const int64_t b = blockIdx.z;
    const int kvh = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.g.kv_heads));
    const int chunk = static_cast<int>(blockIdx.x / static_cast<unsigned>(a.g.kv_heads));
    const SeqView sv = seq_view(a, b, blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0);
    const int64_t total = static_cast<int64_t>(sv.n) * a.per_kv;      // (query row, head of the group) pairs
    const int64_t first = static_cast<int64_t>(chunk) * F::ROWS;
    if (first >= total) return;
    const int rows = total - first < F::ROWS ? static_cast<int>(total - first) : F::ROWS;
    const int i0 = static_cast<int>(first / a.per_kv), i1 = static_cast<int>((first + rows - 1) / a.per_kv);
    int lo, hi, size, count;
    visible(a, sv, i0, i1, lo, hi);
    pieces(a, lo, hi, 16, size, count);
    const int split = blockIdx.y;
    if (split >= (count > 1 ? count : 1)) return;        // (an empty range still writes zeros)
    const int j_begin = (lo & ~15) + split * size;
    int j_end = j_begin + size;
    if (j_end > hi) j_end = hi;
    const int steps = j_end > j_begin ? (j_end - j_begin + 15) >> 4 : 0;

    uint8_t *ring = smem + warp * F::WARP_BYTES;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + kWarps * F::WARP_BYTES) + warp * STAGES;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
    }
    __syncwarp();

    // ---- the copies of one step: lanes 0 .. 3 issue keys, values and their grids ----
    const int32_t *table = a.table + b * a.table_ld;
    const int64_t part_off = lane == 0 ? 0 : lane == 1 ? cache_v_off(a.g) : lane == 2 ? cache_kg_off(a.g) : cache_vg_off(a.g);
    const int tok_bytes = lane < 2 ? D / 2 : 4 * NG;
    const int part_dst = lane == 0 ? 0 : lane == 1 ? F::CODE_BYTES : 2 * F::CODE_BYTES + (lane == 2 ? 0 : F::GRID_BYTES);
    const int my_steps = steps > warp ? (steps - warp + kWarps - 1) / kWarps : 0;
    unsigned absent = 0u;                                // bit s: stage s holds a step whose page id is out of range
    auto page_of = [&](int k) { return k < my_steps ? table[(j_begin + 16 * (warp + kWarps * k)) >> a.g.page_shift] : 0; };
    auto issue = [&](int k, int32_t page) {
        if (k >= my_steps) return;
        const int s = k % STAGES;
        absent &= ~(1u << s);
        if (static_cast<uint32_t>(page) >= static_cast<uint64_t>(a.g.pages)) {   // its tokens count as not there
            absent |= 1u << s;
            page = 0;
            if (lane == 0) set_error(a.err, ERR_RANGE);
        }
        const int j0 = j_begin + 16 * (warp + kWarps * k);
        const int64_t at = j0 & ((1 << a.g.page_shift) - 1);
        if (lane == 0) mbar_arrive_expect_tx(&full[s], F::STEP_BYTES);
        __syncwarp();
        if (lane < 4)
            bulk_load(ring + s * F::STEP_BYTES + part_dst,
                      a.g.data + (static_cast<int64_t>(page) * a.g.kv_heads + kvh) * a.g.block_bytes + part_off + at * tok_bytes,
                      16 * tok_bytes, &full[s]);
    };
    {
        int32_t pg[STAGES - 1];
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) pg[k] = page_of(k);
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) issue(k, pg[k]);
    }
    int32_t next_page = page_of(STAGES - 1);

    // ---- Q^T fragments: lane (r, t) holds row r's channels 32 w + 8 t .. + 7 of every tile ----
    uint32_t qf[NT][C][4];
    float qs[NT][NG][2];                                 // 2^-24 sum of q over a group, rows 2 t and 2 t + 1
    float mult[NT][2];                                   // scores in log2 units per accumulated unit
    int see_lo[NT][2], see_hi[NT][2];                    // visible tokens of rows 2 t, 2 t + 1
    int all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int rr = 8 * n + r;
        float q[C][8];
        float big = 0.0f;
        const int64_t pr = first + (rr < rows ? rr : 0);
        const int i = static_cast<int>(pr / a.per_kv);
        const int head = kvh * a.per_kv + static_cast<int>(pr - static_cast<int64_t>(i) * a.per_kv);
#pragma unroll
        for (int w = 0; w < C; ++w) {
            load_q8(a, sv.row0 + i, head, 32 * w + 8 * t, q[w]);
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(q[w][e]));
        }
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        // 2^e with big 2^-e in [2^14, 2^15): exponents from the bits (zeros and subnormals keep a finite factor)
        int e = static_cast<int>(__float_as_uint(big) >> 23) - 127 - 14;
        if (e < -126) e = -126;
        if (e > 113) e = 113;                            // inf or NaN: the row becomes NaN below
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
        float sum[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) sum[g] = 0.0f;
#pragma unroll
        for (int w = 0; w < C; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                q[w][k] *= down;
                sum[w / GC] += q[w][k];
            }
            qf[n][w][0] = pack_f16(q[w][0], q[w][1]);
            qf[n][w][1] = pack_f16(q[w][2] * 0.0625f, q[w][3] * 0.0625f);
            qf[n][w][2] = pack_f16(q[w][4], q[w][5]);
            qf[n][w][3] = pack_f16(q[w][6] * 0.0625f, q[w][7] * 0.0625f);
        }
        const float m = a.scale2 * 16777216.0f * up;
        int l0, h0;
        visible(a, sv, i, i, l0, h0);
        all_lo = l0 > all_lo ? l0 : all_lo;
        all_hi = h0 < all_hi ? h0 : all_hi;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float s = sum[g];
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            s *= 5.9604644775390625e-8f;                 // 2^-24
            qs[n][g][0] = __shfl_sync(0xffffffffu, s, 8 * t);
            qs[n][g][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4);
        }
        mult[n][0] = __shfl_sync(0xffffffffu, m, 8 * t);
        mult[n][1] = __shfl_sync(0xffffffffu, m, 8 * t + 4);
        see_lo[n][0] = __shfl_sync(0xffffffffu, l0, 8 * t);
        see_lo[n][1] = __shfl_sync(0xffffffffu, l0, 8 * t + 4);
        see_hi[n][0] = __shfl_sync(0xffffffffu, h0, 8 * t);
        see_hi[n][1] = __shfl_sync(0xffffffffu, h0, 8 * t + 4);
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        const int x = __shfl_xor_sync(0xffffffffu, all_lo, o), y = __shfl_xor_sync(0xffffffffu, all_hi, o);
        all_lo = x > all_lo ? x : all_lo;
        all_hi = y < all_hi ? y : all_hi;
    }

    float o[NT][2 * C][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int k = 0; k < 2 * C; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][k][e] = 0.0f;
        m[n][0] = m[n][1] = kFloor;
        l[n][0] = l[n][1] = 0.0f;
    }

    for (int k = 0; k < my_steps; ++k) {
        const int s = k % STAGES;
        __syncwarp();                                    // every lane has read the stage that is refilled now
        const int32_t page = next_page;
        next_page = page_of(k + STAGES);
        issue(k + STAGES - 1, page);
        if (!mbar_wait_bounded(&full[s], (k / STAGES) & 1u, nullptr)) {
            if (lane == 0) set_error(a.err, ERR_TIMEOUT);
            const int last = k + STAGES < my_steps ? k + STAGES : my_steps;
            for (int d = k + 1; d < last; ++d) mbar_wait_bounded(&full[d % STAGES], (d / STAGES) & 1u, nullptr);
            break;
        }
        const uint8_t *st = ring + s * F::STEP_BYTES;
        const int j0 = j_begin + 16 * (warp + kWarps * k);
        const bool gone = (absent >> s) & 1u;
        const bool edge = gone || j0 < all_lo || j0 + 16 > all_hi;

        // ---- scores S^T[token][row] of tokens j0 + r, j0 + r + 8 and rows 2 t, 2 t + 1 ----
        float x[NT][4];
        {
            uint32_t w0[C], w1[C], g0[NG], g1[NG];
            lds_words<C>(st + lane * 4 * C, w0);
            lds_words<C>(st + 4 * D + lane * 4 * C, w1);
            lds_words<NG>(st + 2 * F::CODE_BYTES + r * 4 * NG, g0);
            lds_words<NG>(st + 2 * F::CODE_BYTES + (r + 8) * 4 * NG, g1);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float s0 = __uint_as_float(g0[g] & 0xFFFF0000u), z0 = __uint_as_float(g0[g] << 16);
                const float s1 = __uint_as_float(g1[g] & 0xFFFF0000u), z1 = __uint_as_float(g1[g] << 16);
                float acc[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    acc[n][0] = -z0 * qs[n][g][0];
                    acc[n][1] = -z0 * qs[n][g][1];
                    acc[n][2] = -z1 * qs[n][g][0];
                    acc[n][3] = -z1 * qs[n][g][1];
                }
#pragma unroll
                for (int w = g * GC; w < (g + 1) * GC; ++w) {
                    const uint32_t u0 = w0[w] >> 8, u1 = w1[w] >> 8;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_f16(acc[n], w0[w] & 0x000f000fu, w1[w] & 0x000f000fu, w0[w] & 0x00f000f0u, w1[w] & 0x00f000f0u,
                                qf[n][w][0], qf[n][w][1]);
                        mma_f16(acc[n], u0 & 0x000f000fu, u1 & 0x000f000fu, u0 & 0x00f000f0u, u1 & 0x00f000f0u,
                                qf[n][w][2], qf[n][w][3]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    x[n][0] = fmaf(s0, acc[n][0], x[n][0]);
                    x[n][1] = fmaf(s0, acc[n][1], x[n][1]);
                    x[n][2] = fmaf(s1, acc[n][2], x[n][2]);
                    x[n][3] = fmaf(s1, acc[n][3], x[n][3]);
                }
            }
        }
        bool above = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[n][e] *= mult[n][e & 1];
                if (edge) {
                    const int j = j0 + r + 8 * (e >> 1);
                    if (gone || j < see_lo[n][e & 1] || j >= see_hi[n][e & 1]) x[n][e] = -CUDART_INF_F;
                }
                above = above || x[n][e] > m[n][e & 1] + kRaise;
            }
        }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float top = fmaxf(x[n][c], x[n][c + 2]);
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    top = fmaxf(top, m[n][c]);
                    const float f = ex2(m[n][c] - top);
                    m[n][c] = top;
                    l[n][c] *= f;
#pragma unroll
                    for (int q = 0; q < 2 * C; ++q) {
                        o[n][q][c] *= f;
                        o[n][q][c + 2] *= f;
                    }
                }
            }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[n][e] = ex2(x[n][e] - m[n][e & 1]);
                l[n][e & 1] += x[n][e];
            }
            pf[n][0] = movmatrix_trans(pack_bf16(x[n][0], x[n][1]));
            pf[n][1] = movmatrix_trans(pack_bf16(x[n][2], x[n][3]));
        }

        // ---- O^T[channel][row] += V^T P^T, tokens j0 + 2 t, + 1 and the same 8 further ----
        {
            uint32_t w0[C], w1[C], g0[2 * NG], g1[2 * NG];
            lds_words<C>(st + F::CODE_BYTES + lane * 4 * C, w0);
            lds_words<C>(st + F::CODE_BYTES + 4 * D + lane * 4 * C, w1);
            lds_words<2 * NG>(st + 2 * F::CODE_BYTES + F::GRID_BYTES + 2 * t * 4 * NG, g0);
            lds_words<2 * NG>(st + 2 * F::CODE_BYTES + F::GRID_BYTES + (2 * t + 8) * 4 * NG, g1);
            if (edge) {   // tokens that no row sees may never have been written: nothing of them is used
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = j0 + 2 * t + e;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        if (gone || j < lo || j >= hi) g0[e * NG + g] = 0u;
                        if (gone || j + 8 < lo || j + 8 >= hi) g1[e * NG + g] = 0u;
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const uint32_t s0 = __byte_perm(g0[g], g0[NG + g], 0x7632), s1 = __byte_perm(g1[g], g1[NG + g], 0x7632);
                const uint32_t z0 = add_bf16x2(__byte_perm(g0[g], g0[NG + g], 0x5410), 0x43004300u);   // 128 + z
                const uint32_t z1 = add_bf16x2(__byte_perm(g1[g], g1[NG + g], 0x5410), 0x43004300u);
#pragma unroll
                for (int w = g * GC; w < (g + 1) * GC; ++w) {
                    uint32_t v0[4], v1[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {        // 128 + c in bf16, less 128 + z, times s
                        v0[i] = mul_bf16x2(sub_bf16x2(((w0[w] >> (4 * i)) & 0x000f000fu) | 0x43004300u, z0), s0);
                        v1[i] = mul_bf16x2(sub_bf16x2(((w1[w] >> (4 * i)) & 0x000f000fu) | 0x43004300u, z1), s1);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_bf16(o[n][2 * w], v0[0], v0[1], v1[0], v1[1], pf[n][0], pf[n][1]);
                        mma_bf16(o[n][2 * w + 1], v0[2], v0[3], v1[2], v1[3], pf[n][0], pf[n][1]);
                    }
                }
            }
        }
    }

    // ---- the warps meet: O, m and l of each in its own ring ----
    __syncwarp();
    float *ow = reinterpret_cast<float *>(ring);
    float *mw = ow + F::ROWS * (D + 4), *lw = mw + F::ROWS;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float sum = l[n][c];
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            const int row = 8 * n + 2 * t + c;
            if (r == 0) {
                mw[row] = m[n][c];
                lw[row] = sum;
            }
#pragma unroll
            for (int w = 0; w < C; ++w)
                *reinterpret_cast<float4 *>(ow + row * (D + 4) + 32 * w + 4 * r) =
                    make_float4(o[n][2 * w][c], o[n][2 * w][c + 2], o[n][2 * w + 1][c], o[n][2 * w + 1][c + 2]);
        }
    }
    __syncthreads();
    const int64_t pairs = a.rows * a.q_heads;
    for (int i = threadIdx.x; i < rows * (D / 4); i += kWarps * 32) {
        const int row = i / (D / 4), d = 4 * (i % (D / 4));
        float big = kFloor, sum = 0.0f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            big = fmaxf(big, reinterpret_cast<const float *>(smem + w * F::WARP_BYTES)[F::ROWS * (D + 4) + row]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float *from = reinterpret_cast<const float *>(smem + w * F::WARP_BYTES);
            const float f = ex2(from[F::ROWS * (D + 4) + row] - big);
            const float4 u = *reinterpret_cast<const float4 *>(from + row * (D + 4) + d);
            sum = fmaf(f, from[F::ROWS * (D + 4) + F::ROWS + row], sum);
            v.x = fmaf(f, u.x, v.x);
            v.y = fmaf(f, u.y, v.y);
            v.z = fmaf(f, u.z, v.z);
            v.w = fmaf(f, u.w, v.w);
        }
        if (d >= a.g.dim) continue;
        const int64_t pr = first + row;
        const int64_t qrow = sv.row0 + pr / a.per_kv;
        const int head = kvh * a.per_kv + static_cast<int>(pr % a.per_kv);
        if (count > 1) {
            const int64_t at = split * pairs + qrow * a.q_heads + head;
            *reinterpret_cast<float4 *>(a.part + at * a.g.dim + d) = v;
            if (d == 0) *reinterpret_cast<float2 *>(a.part + a.splits * pairs * a.g.dim + 2 * at) = make_float2(big, sum);
        } else {
            finish(a, qrow, head, d, v, big, sum);
        }
    }
}

// Joins the pieces of each (query row, head): a warp each.
__global__ void __launch_bounds__(256) k_attend_join(const AttendArgs a, int rows_per_chunk, int unit) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t pairs = a.rows * a.q_heads;
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (at >= pairs) return;
    const int64_t qrow = at / a.q_heads;
    const int head = static_cast<int>(at - qrow * a.q_heads);
    // the sequence of this row: the last one that starts at or before it
    int64_t b0 = 0, b1 = a.seqs;
    while (b1 - b0 > 1) {
        const int64_t mid = (b0 + b1) >> 1;
        if (a.q_start[mid] <= qrow) b0 = mid;
        else b1 = mid;
    }
    const SeqView sv = seq_view(a, b0, false);
    const int64_t i = qrow - sv.row0;
    if (i < 0 || i >= sv.n) return;
    const int64_t chunk = (i * a.per_kv + head % a.per_kv) / rows_per_chunk;
    const int64_t first = chunk * rows_per_chunk;
    const int64_t total = static_cast<int64_t>(sv.n) * a.per_kv;
    const int64_t last = (first + rows_per_chunk < total ? first + rows_per_chunk : total) - 1;
    int lo, hi, size, count;
    visible(a, sv, static_cast<int>(first / a.per_kv), static_cast<int>(last / a.per_kv), lo, hi);
    pieces(a, lo, hi, unit, size, count);
    if (count <= 1) return;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part + a.splits * pairs * a.g.dim) + at;
    float big = kFloor;
    for (int s = lane; s < count; s += 32) big = fmaxf(big, ml[s * pairs].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    float sum = 0.0f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const bool mine = 4 * lane < a.g.dim;
    for (int s = 0; s < count; ++s) {
        const float2 q = ml[s * pairs];
        const float f = ex2(q.x - big);
        sum = fmaf(f, q.y, sum);
        if (mine) {
            const float4 u = *reinterpret_cast<const float4 *>(a.part + (s * pairs + at) * a.g.dim + 4 * lane);
            v.x = fmaf(f, u.x, v.x);
            v.y = fmaf(f, u.y, v.y);
            v.z = fmaf(f, u.z, v.z);
            v.w = fmaf(f, u.w, v.w);
        }
    }
    if (mine) finish(a, qrow, head, 4 * lane, v, big, sum);
}

template <int C, int GC, int NT>
cudaError_t launch_rows(const AttendArgs &a, const dim3 &grid, cudaStream_t s) {
    using F = RowsCfg<C, GC, NT>;
    static const cudaError_t once =
        cudaFuncSetAttribute(k_attend_rows<C, GC, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM);
    if (once != cudaSuccess) return once;
    k_attend_rows<C, GC, NT><<<grid, kWarps * 32, F::SMEM, s>>>(a);
    return cudaGetLastError();
}

template <int C, int GC>
cudaError_t launch_rows_nt(const AttendArgs &a, int tiles, const dim3 &grid, cudaStream_t s) {
    if (tiles == 1) return launch_rows<C, GC, 1>(a, grid, s);
    if (tiles == 2) return launch_rows<C, GC, 2>(a, grid, s);
    if constexpr (C == 2) {
        if (tiles == 4) return launch_rows<C, GC, 4>(a, grid, s);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_attend_rows(const AttendArgs &a, int tiles, int64_t row_chunks, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>(row_chunks * a.g.kv_heads), static_cast<unsigned>(a.splits),
                    static_cast<unsigned>(a.seqs));
    const int C = a.g.D / 32, GC = C / a.g.groups;
    if (C == 2) return GC == 1 ? launch_rows_nt<2, 1>(a, tiles, grid, s) : launch_rows_nt<2, 2>(a, tiles, grid, s);
    if (C == 3) return launch_rows_nt<3, 1>(a, tiles, grid, s);
    if (GC == 1) return launch_rows_nt<4, 1>(a, tiles, grid, s);
    if (GC == 2) return launch_rows_nt<4, 2>(a, tiles, grid, s);
    return launch_rows_nt<4, 4>(a, tiles, grid, s);
}

cudaError_t launch_attend_join(const AttendArgs &a, int rows_per_chunk, int unit, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(a.rows * a.q_heads, 8)));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_attend_join, a, rows_per_chunk, unit);
}

}  // namespace qe

using namespace qe;

namespace {

// How a call is cut up: 8-row tiles of a CTA, chunks of rows and pieces of the tokens.
struct AttendPlan {
    int tiles, rows_per_chunk, splits;
    int64_t row_chunks, min_tokens;
};

AttendPlan attend_plan(const CacheGeom &g, int q_heads, int64_t seqs, int64_t max_q, int64_t max_kv) {
    AttendPlan p;
    const int64_t pairs = max_q * (q_heads / g.kv_heads);
    // registers: a tile of 8 rows costs 2 D / 32 accumulators and as much again for Q, so D > 64 takes two at most
    p.tiles = pairs <= 8 ? 1 : (pairs <= 16 || g.D > 64) ? 2 : 4;
    p.rows_per_chunk = 8 * p.tiles;
    p.row_chunks = ceil_div(pairs, p.rows_per_chunk);
    const int64_t ctas = seqs * p.row_chunks * g.kv_heads;
    p.min_tokens = 256;
    int64_t s = ceil_div(152 * 8, ctas);
    const int64_t most = ceil_div(max_kv, p.min_tokens);
    if (s > most) s = most;
    if (s > 128) s = 128;
    p.splits = s < 1 ? 1 : static_cast<int>(s);
    return p;
}

size_t attend_bytes(const AttendPlan &p, const CacheGeom &g, int64_t rows, int q_heads) {
    if (p.splits == 1) return 0;
    return static_cast<size_t>(p.splits) * rows * q_heads * (g.dim + 2) * sizeof(float);
}

// Geometry of a cache that may have no memory yet (the workspace query takes it either way).
qe_status shape_geom(const qe_cache *cache, CacheGeom *g) {
    if (!cache) return QE_ERR_INVALID_ARG;
    qe_cache c = *cache;
    c.data = reinterpret_cast<void *>(static_cast<uintptr_t>(256));
    c.bytes = ~static_cast<size_t>(0);
    return cache_geom(&c, g);
}

qe_status check_shape(const CacheGeom &g, const qe_attention *at) {
    if (!at || at->seqs < 1 || at->rows < 0 || at->q_heads < 1 || at->max_q < 0 || at->max_kv < 0 || at->window < 0)
        return QE_ERR_INVALID_ARG;
    if (at->q_heads % g.kv_heads != 0 || (at->window > 0 && !at->causal)) return QE_ERR_INVALID_ARG;
    if (at->seqs > 65535 || at->rows > (int64_t{1} << 31) - 1 || at->max_q > at->rows || at->max_kv > (1 << 30) ||
        at->window > (int64_t{1} << 31))
        return QE_ERR_INVALID_ARG;
    return QE_OK;
}

}  // namespace

extern "C" {

qe_status qe_cache_attention_workspace(const qe_cache *cache, const qe_attention *at, size_t *bytes) {
    CacheGeom g;
    if (!bytes) return QE_ERR_INVALID_ARG;
    qe_status st = shape_geom(cache, &g);
    if (st != QE_OK) return st;
    if ((st = check_shape(g, at)) != QE_OK) return st;
    *bytes = attend_bytes(attend_plan(g, at->q_heads, at->seqs, at->max_q, at->max_kv), g, at->rows, at->q_heads);
    return QE_OK;
}

qe_status qe_cache_attention(const qe_cache *cache, const qe_attention *at, const void *Q, int64_t q_row, int64_t q_head,
                             void *out, int64_t o_row, int64_t o_head, qe_dtype dtype, float *lse, void *workspace,
                             size_t workspace_bytes, qe_stream_t stream) {
    AttendArgs a{};
    qe_status st = cache_geom(cache, &a.g);
    if (st != QE_OK) return st;
    if ((st = check_shape(a.g, at)) != QE_OK) return st;
    if (dtype != QE_BF16 && dtype != QE_F16) return dtype == QE_F32 ? QE_ERR_UNSUPPORTED : QE_ERR_INVALID_ARG;
    if (at->rows == 0 || at->max_q == 0) return QE_OK;
    if (!at->q_start || !at->kv_len || !at->page_table || at->table_ld < 1 || !Q || !out) return QE_ERR_INVALID_ARG;
    if (at->table_ld > (int64_t{1} << 30) >> a.g.page_shift && at->table_ld << a.g.page_shift > (int64_t{1} << 30))
        return QE_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(out)) & 1u) != 0 ||
        ((reinterpret_cast<uintptr_t>(at->q_start) | reinterpret_cast<uintptr_t>(at->kv_len) |
          reinterpret_cast<uintptr_t>(at->page_table) | reinterpret_cast<uintptr_t>(lse)) & 3u) != 0 ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
        return QE_ERR_INVALID_ARG;
    if (!(at->scale >= 0.0f) || at->scale > 1e30f) return QE_ERR_INVALID_ARG;
    a.q_start = at->q_start;
    a.kv_len = at->kv_len;
    a.table = at->page_table;
    a.table_ld = at->table_ld;
    a.rows = at->rows;
    a.seqs = at->seqs;
    a.max_q = at->max_q;
    a.q_heads = at->q_heads;
    a.per_kv = at->q_heads / a.g.kv_heads;
    a.causal = at->causal != 0;
    a.window = at->window;
    a.scale2 = (at->scale > 0.0f ? at->scale : 1.0f / sqrtf(static_cast<float>(a.g.dim))) * 1.44269504088896341f;
    a.Q = Q;
    a.out = out;
    a.q_row = q_row;
    a.q_head = q_head;
    a.o_row = o_row;
    a.o_head = o_head;
    a.half = dtype == QE_F16;
    a.q_vec = (reinterpret_cast<uintptr_t>(Q) & 15u) == 0 && q_row % 8 == 0 && q_head % 8 == 0;
    a.lse = lse;
    a.err = device_error_word();
    if (!a.err) return QE_ERR_CUDA;
    const AttendPlan p = attend_plan(a.g, at->q_heads, at->seqs, at->max_q, at->max_kv);
    a.splits = p.splits;
    a.min_tokens = p.min_tokens;
    if (p.row_chunks * a.g.kv_heads > 0x7fffffff) return QE_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const size_t need = attend_bytes(p, a.g, at->rows, at->q_heads);
    void *own = nullptr;
    if (need > 0) {
        if (workspace) {
            if (workspace_bytes < need) return QE_ERR_OOM;
            a.part = static_cast<float *>(workspace);
        } else {
            if (cudaMallocAsync(&own, need, s) != cudaSuccess) {
                cudaGetLastError();
                return QE_ERR_OOM;
            }
            a.part = static_cast<float *>(own);
        }
    }
    cudaError_t e = launch_attend_rows(a, p.tiles, p.row_chunks, s);
    if (e == cudaSuccess && p.splits > 1) e = launch_attend_join(a, p.rows_per_chunk, 16, s);
    if (own) cudaFreeAsync(own, s);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return QE_ERR_CUDA;
    }
    return QE_OK;
}

}  // extern "C"
