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
//   values O^T[channel][row] = V^T P^T with c - z, exact in the same subnormals, and
//          P^T's fragment times the scale in fp16, 2^-11 relative: P is rounded before and
//          the product again, which bf16 results do not show; for fp16 ones P's rounding
//          is carried along, so that one is left.
// Grids are turned into what the fragments want once per step by the whole warp and
// read back from shared memory: four lanes of a quad would each do it otherwise.
// Value scales are taken relative to powers of two of their channel groups, whose largest
// P's exponent takes over, and tokens far from the others' size are added by themselves in
// fp32 (qe_attend_out.cuh); the running maximum is raised only when score + e exceeds it
// by 2^8, so accumulators are rarely rescaled.  What a token adds keeps its bits down to
// 2^-21 of the greatest of its row, less up to 2^-7 for its scales within 2^e_g, and
// vanishes 2^10 further down.  Sums and softmax statistics are fp32.
// The 16 x 8 score fragment becomes P^T's fragment by an 8 x 8 transpose in the
// warp.  A warp walks 32-token steps on its own, fed by bulk copies into a ring of
// its own; the warps of a CTA take an item's steps in turn and meet in shared
// memory at the end.  The steps of the whole batch are dealt out evenly over one
// wave of CTAs (ragged lengths, few or many sequences alike), and items that
// fall to several CTAs are joined by a second kernel.
// Measured (whole calls, 32 heads of 128 on 8 unless said): 64 single tokens over 1000
// .. 8191 98 us (3.9 TB/s of cache; moving the bytes alone took 66 .. 75; with one power of
// two for all groups and no tokens apart it was 95), 2 over 128K 74 us (4.0 TB/s), 32 over
// 4K with 232 heads of 64 on 8 70 us: there softmax and operands of 29 rows a kv head bound
// it, not memory.
#pragma once

#include "qe_attend.h"
#include "qe_attend_out.cuh"
#include "qe_internal.h"

namespace qe {
namespace {

// Warps of a CTA.  Two where the steps of the batch are dealt out, so that while the
// warps of one CTA meet and turn to their next item the others of the SM compute (four:
// 64 single tokens over 1K .. 8K 100 us, two: 92); more where a CTA takes a whole item.
constexpr int kDealtWarps = 2;

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

__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
    const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b), *reinterpret_cast<const __half2 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
    const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
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

// CTAs of two warps an SM holds, by registers: 128, 168 and 255 a thread.
__host__ __device__ constexpr int rows_blocks(int C, int NT) { return NT == 1 ? (C == 2 ? 8 : 6) : 4; }

// CTAs of four warps for whole items: three where 168 registers do (16 sequences of 3 .. 5
// rows in a window of 1024, 32 heads of 80: two 34.7 us, three 27.9).
__host__ __device__ constexpr int whole_blocks(int C, int GC, int NT, int warps) { return warps == 4 && NT == 1 && (C < 4 || GC == C) ? 3 : 1; }

// C chunks of 32 channels, GC chunks to a group, NT tiles of 8 query rows.
template <int C, int GC, int NT, int kWarps>
struct RowsCfg {
    static constexpr int D = 32 * C, NG = C / GC, ROWS = 8 * NT;
    static constexpr int CODE_BYTES = 8 * D;              // 16 tokens' key (or value) codes
    static constexpr int GRID_BYTES = 64 * NG;
    static constexpr int STEP_BYTES = 4 * CODE_BYTES + 4 * GRID_BYTES;   // 32 tokens: keys, values, their grids
    static constexpr int STAGES = 2;
    static constexpr int RING = STAGES * STEP_BYTES;      // one warp's
    static constexpr int JOIN = ROWS * (D + 4) * 4 + 2 * ROWS * 4;   // one warp's O, m and l at the end
    static constexpr int KEY_GRIDS = 32 * NG * 8;         // (s, z) of a step's tokens in fp32
    static constexpr int VAL_GRIDS = 16 * NG * 8;         // (s, s'), (z, z') of a step's pairs of tokens in fp16
    static constexpr int APART = 32 * 4 + 32 * ROWS * 4;  // of tokens added by themselves: exponent less e; scores
    static constexpr int USED = RING + KEY_GRIDS + VAL_GRIDS + APART;
    static constexpr int WARP_BYTES = USED > JOIN ? USED : JOIN;
    static constexpr int SMEM = kWarps * WARP_BYTES + kWarps * STAGES * 8 + (kWarps * 32 + 1) * 8;
};

// Adds the tokens `apart` of a step (2 b at bit b, 2 b + 1 at bit 16 + b) to the accumulators in fp32; their scales are
// zero in the fragments.  x: their exponents less e, then all scores with these; the sums have taken P as it is with them.
template <int C, int GC, int NT>
__device__ __forceinline__ void add_apart(const float (&m)[NT][2], float (&l)[NT][2], float (&o)[NT][2 * C][4], unsigned apart, const float *x,
                                          int group_exp, const uint32_t *codes, const uint32_t *grids) {
    const int lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    __syncwarp();
    for (; apart != 0u; apart &= apart - 1u) {
        const int bit = __ffs(static_cast<int>(apart)) - 1, k = 2 * (bit & 15) + (bit >> 4);
        const float back = power(127 - static_cast<int>(x[k]));           // 2^(e - own)
        const uint32_t *words = codes + (k >> 3) * (32 * C) + (4 * r + ((k & 7) >> 1)) * C;
        float p[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                p[n][c] = ex2(x[32 + k * 8 * NT + 8 * n + 2 * t + c] - m[n][c]);
                if (r == 0) l[n][c] = fmaf(p[n][c], back - 1.0f, l[n][c]);
                p[n][c] *= back;
            }
#pragma unroll
        for (int w = 0; w < C; ++w) {
            const int g = w / GC;
            const uint32_t grid = grids[k * (C / GC) + g], code = words[w] >> (16 * (k & 1));
            const float s = __uint_as_float(grid & 0xFFFF0000u), z = __uint_as_float(grid << 16);
            // the accumulators' units, 2^(24 + e_g - e), of channels 4 r + 1 and 4 r + 3 of the chunk 2^4 less, and 2^-e of P
            const float unit = __shfl_sync(0xffffffffu, power(127 + 127 - 24 - group_exp), g);
            auto channel = [&](int i) { return s * (static_cast<float>(code >> (4 * i) & 15u) - z); };
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float pu = p[n][c] * unit, pu4 = pu * 16.0f;
                    o[n][2 * w][c] = fmaf(pu, channel(0), o[n][2 * w][c]);
                    o[n][2 * w][c + 2] = fmaf(pu4, channel(1), o[n][2 * w][c + 2]);
                    o[n][2 * w + 1][c] = fmaf(pu, channel(2), o[n][2 * w + 1][c]);
                    o[n][2 * w + 1][c + 2] = fmaf(pu4, channel(3), o[n][2 * w + 1][c + 2]);
                }
        }
    }
}

// HALF: fp16 queries and results, bf16 otherwise.
// WHOLE: block x takes item x whole (items numbered by the longest sequence), nothing is dealt out or joined.
template <int C, int GC, int NT, int kWarps, bool WHOLE, bool HALF>
__global__ void __launch_bounds__(kWarps * 32, WHOLE ? whole_blocks(C, GC, NT, kWarps) : rows_blocks(C, NT)) k_attend_rows(const AttendArgs a) {
    using F = RowsCfg<C, GC, NT, kWarps>;
    constexpr int D = F::D, NG = F::NG, STAGES = F::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, t = lane & 3;
    uint8_t *ring = smem + warp * F::WARP_BYTES;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + kWarps * F::WARP_BYTES) + warp * STAGES;
    int64_t *sums = reinterpret_cast<int64_t *>(smem + kWarps * F::WARP_BYTES + kWarps * STAGES * 8);
    if constexpr (!WHOLE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
    }
    int64_t share = 0, cta_begin, cta_end;
    Place at;
    at.seq = -1;
    if constexpr (WHOLE) {
        const unsigned of_seq = static_cast<unsigned>(a.items) / static_cast<unsigned>(a.seqs);
        at.seq = blockIdx.x / of_seq;
        at.base = 0;
        at.v = seq_view(a, at.seq, blockIdx.x == at.seq * of_seq && threadIdx.x == 0);
        at.w = seq_work(a, at.v, kRowsUnit);
        cta_begin = static_cast<int64_t>(blockIdx.x - at.seq * of_seq) * at.w.steps;
        if (cta_begin >= at.w.units) return;
        cta_end = cta_begin + at.w.steps;
    } else {
        scan_units<kWarps * 32>(a, kRowsUnit, sums, share);
        const int64_t total_units = sums[kWarps * 32];
        const int64_t per = worker_units(a, total_units);
        cta_begin = blockIdx.x * per;
        cta_end = cta_begin + per < total_units ? cta_begin + per : total_units;
    }

    // lanes 0 .. 7 copy a step: keys, values and their grids of its two halves of 16 tokens
    const int part_of = lane & 3, half_of = (lane >> 2) & 1;
    const uint32_t part_off = part_of == 0 ? 0u : part_of == 1 ? a.g.v_off : part_of == 2 ? a.g.kg_off : a.g.vg_off;
    const int tok_bytes = part_of < 2 ? D / 2 : 4 * NG;
    const int part_dst = part_of == 0 ? half_of * F::CODE_BYTES : part_of == 1 ? (2 + half_of) * F::CODE_BYTES
                         : 4 * F::CODE_BYTES + (part_of == 2 ? half_of : 2 + half_of) * F::GRID_BYTES;
    const bool wide = a.g.page_shift >= 5;                // a step lies in one page: one copy for both halves
    const int page_mask = (1 << a.g.page_shift) - 1;
    unsigned turn = 0;                                    // steps this warp has taken: stage and phase of the next
    bool stuck = false;

    for (int64_t pos = cta_begin; pos < cta_end;) {
        if constexpr (!WHOLE) locate<kWarps * 32>(a, kRowsUnit, sums, share, pos, at);
        const SeqView sv = at.v;
        const int64_t item = div_small(pos - at.base, at.w.steps);
        const int step0 = static_cast<int>(pos - at.base - item * at.w.steps);
        const int64_t left = cta_end - pos;
        const int take = left < at.w.steps - step0 ? static_cast<int>(left) : at.w.steps - step0;
        const int chunk = static_cast<int>(div_small(item, a.g.kv_heads));
        const int kvh = static_cast<int>(item - static_cast<int64_t>(chunk) * a.g.kv_heads);
        const int first = chunk * F::ROWS, all = sv.n * a.per_kv;
        const int rows = all - first < F::ROWS ? all - first : F::ROWS;
        const int lo = at.w.lo, hi = at.w.hi;
        const int j_begin = (lo & ~(kRowsUnit - 1)) + step0 * kRowsUnit;
        const int my_steps = hi > lo && take > warp ? (take - warp + kWarps - 1) / kWarps : 0;
        const int32_t *table = a.table + at.seq * a.table_ld;
        const uint8_t *mine = a.g.data + kvh * a.g.block_bytes + part_off;
        const int64_t page_bytes = a.g.page_bytes;

        unsigned gone = 0u;                               // 2 bits a stage: halves whose page id is out of range
        auto page_of = [&](int k) {                       // (halves without a visible token take the nearest one's page)
            int j = j_begin + kRowsUnit * (warp + kWarps * k) + 16 * half_of;
            j = max(min(j, hi - 1), lo & ~15);
            return k < my_steps ? table[j >> a.g.page_shift] : 0;
        };
        auto issue = [&](int k, int32_t page) {
            if (k >= my_steps) return;
            const int s = (turn + k) % STAGES;
            const bool out = static_cast<uint32_t>(page) >= static_cast<uint64_t>(a.g.pages);
            const unsigned votes = __ballot_sync(0xffffffffu, out);
            gone &= ~(3u << (2 * s));
            if (votes != 0u) {                            // its tokens count as not there
                gone |= ((votes & 1u) | (votes >> 3 & 2u)) << (2 * s);
                if (out) page = 0;
                if (lane == 0) set_error(a.err, ERR_RANGE);
            }
            const int j = j_begin + kRowsUnit * (warp + kWarps * k) + 16 * half_of;
            if (lane == 0) mbar_arrive_expect_tx(&full[s], F::STEP_BYTES);
            __syncwarp();
            if (lane < (wide ? 4 : 8))
                bulk_load(ring + s * F::STEP_BYTES + part_dst, mine + page * page_bytes + (j & page_mask) * tok_bytes,
                          (wide ? 32 : 16) * tok_bytes, &full[s]);
        };
        {
            int32_t pg[STAGES];
#pragma unroll
            for (int k = 0; k < STAGES; ++k) pg[k] = page_of(k);
#pragma unroll
            for (int k = 0; k < STAGES; ++k) issue(k, pg[k]);
        }
        int32_t next_page = page_of(STAGES);

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
            const unsigned pr = first + (rr < rows ? rr : 0);
            const int i = pr / static_cast<unsigned>(a.per_kv);
            const int head = kvh * a.per_kv + static_cast<int>(pr) - i * a.per_kv;
#pragma unroll
            for (int w = 0; w < C; ++w) {
                load_q8(a, sv.row0 + i, head, 32 * w + 8 * t, q[w]);
#pragma unroll
                for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(q[w][e]));
            }
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
            float down, up;
            q_powers(big, down, up);
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
            const float m = fminf(a.scale2 * 16777216.0f * up, 1.70141183e38f);   // (finite: scores may be 0)
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
        float o[NT][2 * C][4];                            // O^T: channels and rows as the fragments have them
        float m[NT][2], l[NT][2];
        constexpr int PER = (16 * NG + 31) / 32;          // (pair of tokens, channel group)s of a lane: lane + 32 i
        int val_exp = kLeastExp;                          // e, and 2^-e_g of these groups
        float down[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) down[i] = power(254 - kLeastExp);
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
            const int s = (turn + k) % STAGES;
            if (!stuck && !mbar_wait_bounded(&full[s], ((turn + k) / STAGES) & 1u, nullptr)) stuck = true;
            const uint8_t *st = ring + s * F::STEP_BYTES;
            const int j0 = j_begin + kRowsUnit * (warp + kWarps * k);
            const unsigned lost = (gone >> (2 * s)) & 3u;
            const bool edge = lost != 0u || j0 < all_lo || j0 + kRowsUnit > all_hi;

            // ---- the step's grids, each turned once ----
            float2 *kgrid = reinterpret_cast<float2 *>(ring + F::RING);
            uint2 *vgrid = reinterpret_cast<uint2 *>(ring + F::RING + F::KEY_GRIDS);
            float *apart_x = reinterpret_cast<float *>(ring + F::RING + F::KEY_GRIDS + F::VAL_GRIDS);
            const uint32_t *kwords = reinterpret_cast<const uint32_t *>(st + 4 * F::CODE_BYTES), *vwords = kwords + 32 * NG;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const uint32_t w = kwords[lane + 32 * i];
                kgrid[lane + 32 * i] = make_float2(__uint_as_float(w & 0xFFFF0000u), __uint_as_float(w << 16));
            }
            auto grids_of = [&](int pair, int g, uint32_t unseen, uint32_t &v0, uint32_t &v1) {
                v0 = vwords[2 * pair * NG + g];
                v1 = vwords[(2 * pair + 1) * NG + g];
                if (edge) {   // grids of tokens that no row sees may never have been written: nothing of them is used
                    const int j = j0 + 2 * pair;
                    const bool none = (lost >> (pair >> 3)) & 1u;
                    if (none || j < lo || j >= hi) v0 = unseen;
                    if (none || j + 1 < lo || j + 1 >= hi) v1 = unseen;
                }
            };
            auto scaled = [&](uint32_t v0, uint32_t v1, float by) {
                return pack_f16(__uint_as_float(v0 & 0xFFFF0000u) * by, __uint_as_float(v1 & 0xFFFF0000u) * by);
            };
            if (k == 0) {                                 // one e for all groups to begin with
                int most = kLeastExp;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int at = lane + 32 * i < 16 * NG ? lane + 32 * i : 16 * NG - 1;
                    uint32_t v0, v1;
                    grids_of(at / NG, at % NG, 0u, v0, v1);
                    most = max(most, max(scale_exp(v0), scale_exp(v1)) + kHeadroom);
                }
                val_exp = min(__reduce_max_sync(0xffffffffu, most), kMostExp);
#pragma unroll
                for (int i = 0; i < PER; ++i) down[i] = power(254 - val_exp);
            }
            uint32_t s2[PER], z2[PER], off = 0u;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = lane + 32 * i < 16 * NG ? lane + 32 * i : 16 * NG - 1;
                uint32_t v0, v1;
                grids_of(at / NG, at % NG, 0x7F000000u - __float_as_uint(down[i]), v0, v1);   // (a scale that fits, 1)
                s2[i] = scaled(v0, v1, down[i]);
                // 128 + z in bf16 ends in z's four bits: the integer, which is z in fp16's units of 2^-24
                z2[i] = add_bf16x2(__byte_perm(v0, v1, 0x5410), 0x43004300u) & 0x000f000fu;
                off |= misfits(s2[i]);
            }
            unsigned apart = 0u;                          // tokens that are added by themselves
            if (__any_sync(0xffffffffu, off != 0u)) {
                constexpr int G2 = (NG + 1) / 2;
                uint32_t w0[G2], w1[G2];
                int eg[G2], before[NG], t0, t1;
                const int val_was = val_exp, eg_was = 254 - static_cast<int>(__float_as_uint(down[0]) >> 23);
#pragma unroll
                for (int g = 0; g < NG; ++g) before[g] = val_exp - __shfl_sync(0xffffffffu, eg_was, g);
#pragma unroll
                for (int i = 0; i < G2; ++i) {
                    grids_of(lane & 15, group_of<NG>(i), 0u, w0[i], w1[i]);
                    eg[i] = __shfl_sync(0xffffffffu, eg_was, group_of<NG>(i));
                }
                apart = refit(w0, w1, val_exp, eg, t0, t1);
#pragma unroll
                for (int g = 0; g < NG; ++g) {            // accumulators are in units of 2^(e_g - e)
                    const int now = __shfl_sync(0xffffffffu, eg[g / 2], 16 * (g & 1));
                    const float f = power(127 + val_exp - now - before[g]);
#pragma unroll
                    for (int i = 0; i < PER; ++i)
                        if ((lane + 32 * i < 16 * NG ? lane + 32 * i : 16 * NG - 1) % NG == g) down[i] = power(254 - now);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int q = 2 * g * GC; q < 2 * (g + 1) * GC; ++q)
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[n][q][c] *= f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)              // maxima less e, sums times 2^e
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        m[n][c] -= static_cast<float>(val_exp - val_was);
                        l[n][c] *= power(127 + val_exp - val_was);
                    }
                if (lane < 16) {
                    apart_x[2 * lane] = static_cast<float>(apart >> lane & 1u ? t0 - val_exp : 0);
                    apart_x[2 * lane + 1] = static_cast<float>(apart >> lane & 0x10000u ? t1 - val_exp : 0);
                }
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int at = lane + 32 * i < 16 * NG ? lane + 32 * i : 16 * NG - 1;
                    uint32_t v0, v1;
                    grids_of(at / NG, at % NG, 0u, v0, v1);
                    s2[i] = scaled(apart >> (at / NG) & 1u ? 0u : v0, apart >> (at / NG) & 0x10000u ? 0u : v1, down[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (16 * NG % 32 == 0 || lane + 32 * i < 16 * NG) vgrid[lane + 32 * i] = make_uint2(s2[i], z2[i]);
            __syncwarp();

#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                // ---- scores S^T[token][row]: tokens j0 + 16 h + r and 8 further, rows 2 t, 2 t + 1 ----
                float x[NT][4];
                {
                    uint32_t w0[C], w1[C], g0[2 * NG], g1[2 * NG];
                    const uint8_t *codes = st + h * F::CODE_BYTES + lane * 4 * C;
                    lds_words<C>(codes, w0);
                    lds_words<C>(codes + 4 * D, w1);
                    const uint8_t *grids = reinterpret_cast<const uint8_t *>(kgrid) + (16 * h + r) * 8 * NG;
                    lds_words<2 * NG>(grids, g0);
                    lds_words<2 * NG>(grids + 64 * NG, g1);
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const float s0 = __uint_as_float(g0[2 * g]), z0 = __uint_as_float(g0[2 * g + 1]);
                        const float s1 = __uint_as_float(g1[2 * g]), z1 = __uint_as_float(g1[2 * g + 1]);
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
                                mma_f16(acc[n], w0[w] & 0x000f000fu, w1[w] & 0x000f000fu, w0[w] & 0x00f000f0u,
                                        w1[w] & 0x00f000f0u, qf[n][w][0], qf[n][w][1]);
                                mma_f16(acc[n], u0 & 0x000f000fu, u1 & 0x000f000fu, u0 & 0x00f000f0u, u1 & 0x00f000f0u,
                                        qf[n][w][2], qf[n][w][3]);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            x[n][0] = g == 0 ? s0 * acc[n][0] : fmaf(s0, acc[n][0], x[n][0]);
                            x[n][1] = g == 0 ? s0 * acc[n][1] : fmaf(s0, acc[n][1], x[n][1]);
                            x[n][2] = g == 0 ? s1 * acc[n][2] : fmaf(s1, acc[n][2], x[n][2]);
                            x[n][3] = g == 0 ? s1 * acc[n][3] : fmaf(s1, acc[n][3], x[n][3]);
                        }
                    }
                }
                bool above = false;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][e] *= mult[n][e & 1];
                }
                if (edge || apart) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = j0 + 16 * h + r + 8 * (e >> 1);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (((lost >> h) & 1u) || j < see_lo[n][e & 1] || j >= see_hi[n][e & 1]) x[n][e] = -CUDART_INF_F;
                    }
                    if (apart) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int k = 16 * h + r + 8 * (e >> 1);
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                x[n][e] += apart_x[k];
                                apart_x[32 + k * F::ROWS + 8 * n + 2 * t + (e & 1)] = x[n][e];
                            }
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) above = above || fmaxf(x[n][c], x[n][c + 2]) > m[n][c] + (kAbove + kRaise);
                if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float u = fmaxf(x[n][c], x[n][c + 2]);
                            u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, 4));
                            u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, 8));
                            u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, 16));
                            u = fmaxf(u - kAbove, m[n][c]);
                            const float f = ex2(m[n][c] - u);
                            m[n][c] = u;
                            l[n][c] *= f;
#pragma unroll
                            for (int q = 0; q < 2 * C; ++q) {
                                o[n][q][c] *= f;
                                o[n][q][c + 2] *= f;
                            }
                        }
                    }
                }
                uint32_t pf[NT][2], pl[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[n][e] = ex2(x[n][e] - m[n][e & 1]);
                        l[n][e & 1] += x[n][e];
                    }
                    pf[n][0] = pack_f16(x[n][0], x[n][1]);
                    pf[n][1] = pack_f16(x[n][2], x[n][3]);
                    if constexpr (HALF) {                 // what the rounding left out
                        const __half2 h0 = *reinterpret_cast<const __half2 *>(&pf[n][0]), h1 = *reinterpret_cast<const __half2 *>(&pf[n][1]);
                        pl[n][0] = movmatrix_trans(pack_f16(x[n][0] - __low2float(h0), x[n][1] - __high2float(h0)));
                        pl[n][1] = movmatrix_trans(pack_f16(x[n][2] - __low2float(h1), x[n][3] - __high2float(h1)));
                    }
                    pf[n][0] = movmatrix_trans(pf[n][0]);
                    pf[n][1] = movmatrix_trans(pf[n][1]);
                }
                // ---- O^T[channel][row] += (c - z)^T (P s)^T over tokens 2 t, 2 t + 1 and the same 8 further ----
                uint32_t w0[C], w1[C], g0[2 * NG], g1[2 * NG];
                const uint8_t *codes = st + (2 + h) * F::CODE_BYTES + lane * 4 * C;
                lds_words<C>(codes, w0);
                lds_words<C>(codes + 4 * D, w1);
                const uint8_t *grids = reinterpret_cast<const uint8_t *>(vgrid) + (8 * h + t) * 8 * NG;
                lds_words<2 * NG>(grids, g0);
                lds_words<2 * NG>(grids + 32 * NG, g1);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    uint32_t ps[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (HALF) {
                            ps[n][0] = fma_f16x2(pf[n][0], g0[2 * g], mul_f16x2(pl[n][0], g0[2 * g]));
                            ps[n][1] = fma_f16x2(pf[n][1], g1[2 * g], mul_f16x2(pl[n][1], g1[2 * g]));
                        } else {
                            ps[n][0] = mul_f16x2(pf[n][0], g0[2 * g]);
                            ps[n][1] = mul_f16x2(pf[n][1], g1[2 * g]);
                        }
                    }
                    const uint32_t z0 = g0[2 * g + 1], z1 = g1[2 * g + 1];
                    const uint32_t y0 = mul_f16x2(z0, 0x4C004C00u), y1 = mul_f16x2(z1, 0x4C004C00u);   // 16 z
#pragma unroll
                    for (int w = g * GC; w < (g + 1) * GC; ++w) {
                        // channels 4 r and 4 r + 2 of the chunk come out in units of 2^-24, 4 r + 1 and 4 r + 3 of 2^-20
                        const uint32_t u0 = w0[w] >> 8, u1 = w1[w] >> 8;
                        const uint32_t v[8] = {sub_f16x2(w0[w] & 0x000f000fu, z0), sub_f16x2(w0[w] & 0x00f000f0u, y0),
                                               sub_f16x2(w1[w] & 0x000f000fu, z1), sub_f16x2(w1[w] & 0x00f000f0u, y1),
                                               sub_f16x2(u0 & 0x000f000fu, z0),    sub_f16x2(u0 & 0x00f000f0u, y0),
                                               sub_f16x2(u1 & 0x000f000fu, z1),    sub_f16x2(u1 & 0x00f000f0u, y1)};
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma_f16(o[n][2 * w], v[0], v[1], v[2], v[3], ps[n][0], ps[n][1]);
                            mma_f16(o[n][2 * w + 1], v[4], v[5], v[6], v[7], ps[n][0], ps[n][1]);
                        }
                    }
                }
            }
            if (apart)
                add_apart<C, GC, NT>(m, l, o, apart, apart_x, 254 - static_cast<int>(__float_as_uint(down[0]) >> 23),
                                     reinterpret_cast<const uint32_t *>(st + 2 * F::CODE_BYTES), vwords);
            __syncwarp();                                 // every lane has read the stage: refill it
            const int32_t page = next_page;
            next_page = page_of(k + STAGES + 1);
            issue(k + STAGES, page);
        }
        turn += my_steps;

        // ---- the warps meet: O, m and l of each in its own ring ----
        __syncwarp();
        float unit[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g)
            unit[g] = __shfl_sync(0xffffffffu, power(127 + 24 + 254 - static_cast<int>(__float_as_uint(down[0]) >> 23) - val_exp), g);
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
                    mw[row] = m[n][c] + static_cast<float>(val_exp - 127);
                    lw[row] = sum * power(254 - val_exp);
                }
#pragma unroll
                for (int w = 0; w < C; ++w) {
                    const float u = unit[w / GC], u4 = u * 0.0625f;
                    *reinterpret_cast<float4 *>(ow + row * (D + 4) + 32 * w + 4 * r) =
                        make_float4(o[n][2 * w][c] * u, o[n][2 * w][c + 2] * u4, o[n][2 * w + 1][c] * u, o[n][2 * w + 1][c + 2] * u4);
                }
            }
        }
        __syncthreads();
        const bool whole = WHOLE || take == at.w.steps;
        float *slot = a.part + (2 * static_cast<int64_t>(blockIdx.x) + (step0 == 0 ? 1 : 0)) * (F::ROWS * (D + 2));
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
            if (!whole) {
                *reinterpret_cast<float4 *>(slot + row * D + d) = v;
                if (d == 0) {
                    slot[F::ROWS * D + row] = big;
                    slot[F::ROWS * (D + 1) + row] = sum;
                }
            } else if (d < a.g.dim) {
                const unsigned pr = first + row, i = pr / static_cast<unsigned>(a.per_kv);
                finish(a, sv.row0 + i, kvh * a.per_kv + static_cast<int>(pr - i * a.per_kv), d, v, big, sum);
            }
        }
        pos += take;
        if (pos < cta_end) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the ring takes copies again
            __syncthreads();
        }
    }
    if (stuck) {                                          // a wait gave up: leave no copy in flight behind
        for (unsigned s = 0; s < STAGES && s < turn; ++s) {
            const unsigned last = turn - 1 - (turn - 1 - s) % STAGES;
            mbar_wait_bounded(&full[s], (last / STAGES) & 1u, nullptr);
        }
        if (lane == 0) set_error(a.err, ERR_TIMEOUT);
    }
}

template <int C, int GC, int NT, int W, bool WHOLE, bool HALF>
cudaError_t launch_rows_as(const AttendArgs &a, cudaStream_t s) {
    using F = RowsCfg<C, GC, NT, W>;
    static std::atomic<uint64_t> raised{0};
    const cudaError_t e = raise_smem(reinterpret_cast<const void *>(k_attend_rows<C, GC, NT, W, WHOLE, HALF>), F::SMEM, raised);
    if (e != cudaSuccess) return e;
    k_attend_rows<C, GC, NT, W, WHOLE, HALF><<<static_cast<unsigned>(WHOLE ? a.items : a.ctas), W * 32, F::SMEM, s>>>(a);
    return cudaGetLastError();
}

template <int C, int GC, int NT, int W, bool WHOLE>
cudaError_t launch_rows(const AttendArgs &a, cudaStream_t s) {
    return a.half ? launch_rows_as<C, GC, NT, W, WHOLE, true>(a, s) : launch_rows_as<C, GC, NT, W, WHOLE, false>(a, s);
}

template <int C, int GC, int W, bool WHOLE>
cudaError_t launch_rows_nt(const AttendArgs &a, int tiles, cudaStream_t s) {
    if (tiles == 1) return launch_rows<C, GC, 1, W, WHOLE>(a, s);
    if (tiles == 2) return launch_rows<C, GC, 2, W, WHOLE>(a, s);
    if constexpr (C == 2) {
        if (tiles == 4) return launch_rows<C, GC, 4, W, WHOLE>(a, s);
    }
    return cudaErrorInvalidValue;
}

template <int W, bool WHOLE>
cudaError_t launch_rows_any(const AttendArgs &a, int tiles, cudaStream_t s) {
    const int C = a.g.D / 32, GC = C / a.g.groups;
    if (C == 2) return GC == 1 ? launch_rows_nt<2, 1, W, WHOLE>(a, tiles, s) : launch_rows_nt<2, 2, W, WHOLE>(a, tiles, s);
    if (C == 3) return launch_rows_nt<3, 1, W, WHOLE>(a, tiles, s);
    if (GC == 1) return launch_rows_nt<4, 1, W, WHOLE>(a, tiles, s);
    return GC == 2 ? launch_rows_nt<4, 2, W, WHOLE>(a, tiles, s) : launch_rows_nt<4, 4, W, WHOLE>(a, tiles, s);
}

}  // namespace
}  // namespace qe
