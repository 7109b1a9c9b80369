// Attention over the 4-bit key/value cache, many query rows per kv head (chunks of
// prompts, whole prompts): the fifth-generation tensor cores, codes turned into
// operands on the way.
//
// A CTA takes 256 (query row, head) pairs that read one kv head, as two tiles of
// 128 rows, and walks its visible tokens in steps of 128.  Bound by the tensor
// cores' 4 x 128^2 x D products a step and, nearly as much, by issuing what
// softmax (256 x 128 exponentials) and the turning of 2 x 128 x D codes cost; two
// row tiles share each turned step.  Roles:
//   warps 0-15       softmax, a thread a row and 64 tokens of the step: warps 0-3 and
//                    8-11 have row tile 0, 4-7 and 12-15 tile 1.  Scores come from tensor
//                    memory into registers, P goes back in their place as the A operand
//                    of the second product;
//   warps 16-19      key codes to fp16 operands [token][channel] in shared memory
//                    (128-byte swizzle), warps 20-23 value codes to [channel][token];
//                    the next step's codes are loaded while the products run;
//   warp 24          issues the products, one tile's while softmax is at the other's.  (A
//                    thread of the softmax warps that issued them itself was held by the
//                    filled tensor queue.)
// What was measured on the way, a causal prompt of 8192 tokens, 32 heads of 128 on 32:
// scores of 64 tokens a product, two buffers a row tile, four softmax warps a tile 568
// us (a product of 128 x 64 takes as long as one of 128 x 128); whole steps and eight
// warps a tile 540; exponentials taken at the old maximum before the new scores' is
// known 512; tokens that may sit out a step 528, which is 1.04 PFLOP/s (with such tokens
// added in fp32 by the softmax warps 598, for want of registers).  The tensor pipe is active
// less than half of the time: the rest is the chain scores - softmax - P - products of
// either row tile.
// Numerics: K' = s (c - z) 2^-F and V' = s (c - z) 2^-E are rounded once to fp16, with
// powers of two for each 32 tokens that bring the largest key scale to 2^10 and a token's
// largest value scale to 2^-2 .. 2^10, so that scales of other tokens and channel groups keep
// their bits down to 2^-14; Q's rows likewise.  2^F and the row's power of two go into
// the score's multiplier, E into the exponent of P and 2^-E into the row sum.  Tokens whose
// values do not fit the others' power of two sit out, and the step is taken again with
// them and an E of theirs (seldom).  The running maximum is one of score + E, of what a token
// adds, and raised only when one exceeds it by 8 (a factor of 2^8), so the accumulator in
// tensor memory is rarely rescaled; P is taken 2^7 above it, keeps its bits down to 2^-21
// of the greatest and vanishes 2^10 further down.  Sums are fp32.
#include <cuda_fp16.h>
#include <math_constants.h>

#include "qe_attend.h"
#include "qe_attend_out.cuh"
#include "qe_internal.h"

namespace qe {
namespace {

constexpr int kTile = 128;                // rows of a tile, tokens of a step
constexpr int kHalf = 64;                 // tokens of a step that a softmax warp takes
constexpr int kThreads = 896;             // the last three warps have no part in it
constexpr int kKeyWarp = 16, kValWarp = 20, kMmaWarp = 24;
constexpr int kKeyRoom = 10, kValRoom = 10;   // log2 of the power of two that the largest scale is brought to
constexpr int kTileWindow = 12;           // log2 of how far below it a token's largest value scale may be
constexpr int kLeastE = 127 - 80;         // E + kValRoom is not below this: with 2^90 the sum of P stays finite
constexpr int kInfos = 4;                // the turning warps are at most two steps ahead of softmax

// Issued by one elected lane of a warp that goes along together, so that addresses stay in
// uniform registers.
__device__ __forceinline__ void mma_ts_one(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void mma_ss_one(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void commit_one(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(bar)
        : "memory");
}

__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, float (&v)[16]) {
    asm volatile(
        "{\n\ttcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t}"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr)
        : "memory");
}

template <class T>
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const T (&v)[16]) {
    static_assert(sizeof(T) == 4, "32 bits a column");
    uint32_t r[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) memcpy(&r[e], &v[e], 4);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// Two warps meet at named barrier `id`.
__device__ __forceinline__ void sync_64(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
// They meet and learn whether any of them says so.
__device__ __forceinline__ bool any_of_64(int id, bool mine) {
    int any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbar.red.or.pred p, %2, 64, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
        : "=r"(any) : "r"(static_cast<int>(mine)), "r"(id) : "memory");
    return any != 0;
}

__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2 *>(&w); }

// (x, y) * k + b and sums, two at a time
__device__ __forceinline__ void fma2(float &x, float &y, uint64_t k, uint64_t b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(v) : "l"(k), "l"(b));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ uint64_t twice(float x) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %1};" : "=l"(v) : "f"(x));
    return v;
}
__device__ __forceinline__ void add2(uint64_t &s, float x, float y) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(s) : "l"(v));
}

__device__ __forceinline__ float total(const uint64_t (&s)[4]) {
    uint64_t v;
    asm("{\n\t.reg .b64 t;\n\tadd.rn.f32x2 t, %1, %2;\n\tadd.rn.f32x2 %0, %3, %4;\n\tadd.rn.f32x2 %0, %0, t;\n\t}"
        : "=&l"(v) : "l"(s[0]), "l"(s[1]), "l"(s[2]), "l"(s[3]));
    float x, y;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
    return x + y;
}

// The warps that turn codes meet and learn whether any of them says so.
__device__ __forceinline__ bool any_turning(bool mine) {
    int any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbar.red.or.pred p, 11, 256, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
        : "=r"(any) : "r"(static_cast<int>(mine)) : "memory");
    return any != 0;
}

// Whether a token whose largest value scale has exponent b (biased; 0, 1: unseen, all zeros or marked bad, no matter) does not fit.
__device__ __forceinline__ bool misfit(int b, int e) { return b > e || (b > 1 && b < e - kTileWindow && e > kLeastE); }

// Of the tokens `left` of 32, b the exponent of the lane's: a new e that at least a quarter of them fit; those that do not.
__device__ __forceinline__ unsigned refit_tokens(int b, unsigned left, int &e) {
    const int lane = threadIdx.x & 31;
    unsigned rest = left & __ballot_sync(0xffffffffu, b > 1);
    const int n = __popc(rest);
    while (true) {
        e = __reduce_max_sync(0xffffffffu, (rest >> lane & 1u) ? b : 0);
        const unsigned in = rest & __ballot_sync(0xffffffffu, b >= e - (kTileWindow - kHeadroom));
        rest &= ~in;
        if (4 * __popc(in) >= n || rest == 0u) break;
    }
    e = max(e + kHeadroom, kLeastE);
    return left & __ballot_sync(0xffffffffu, misfit(b, e));
}

__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// What the softmax warps need to know of a turned step.
struct StepInfo {
    float key_up[4];          // 2^F of 32 tokens each
    float val_exp[4];         // E
    float val_down[4];        // 2^-E
    unsigned out[4];          // of each 32 tokens, those that sit out
    int step;                 // which step of the item it is; negative (and one less): the last one
    uint8_t gone[4];          // of each 32 tokens, a bit for either 16, their page id is out of range; 4: some sit out
};

template <int C, int GC>
struct TcCfg {
    static constexpr int D = 32 * C, NG = C / GC, DQ = D <= 64 ? 64 : 128;   // DQ: channels in whole swizzle atoms of 64
    static constexpr int Q_BYTES = kTile * DQ * 2;        // one row tile
    static constexpr int K_BYTES = kTile * DQ * 2;
    static constexpr int V_BYTES = D * kTile * 2;
    static constexpr int VPAIRS = 4 * 16 * NG * 8;        // (s, s'), (z, z') of the step's pairs of tokens
    static constexpr int BAR_OFF = 2 * Q_BYTES + 2 * K_BYTES + 2 * V_BYTES + VPAIRS;
    static constexpr int ROW_OFF = BAR_OFF + 20 * 8 + kInfos * static_cast<int>(sizeof(StepInfo));   // floats of the rows
    static constexpr int SMEM = 1024 + ROW_OFF + 5 * 2 * kTile * 4;
    // one CTA an SM: it takes all of tensor memory
    static constexpr int SMEM_ASKED = SMEM > 120 * 1024 ? SMEM : 120 * 1024;
};

template <int C, int GC>
__global__ void __launch_bounds__(kThreads, 1) k_attend_tiles(const AttendArgs a) {
    using F = TcCfg<C, GC>;
    constexpr int D = F::D, NG = F::NG;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t pad = (1024u - (smem_u32(smem_raw) & 1023u)) & 1023u;
    uint8_t *smem = smem_raw + pad;
    uint8_t *sq = smem, *sk = sq + 2 * F::Q_BYTES, *sv_ = sk + 2 * F::K_BYTES, *spairs = sv_ + 2 * F::V_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + F::BAR_OFF);
    uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6;
    uint64_t *s_full = bars + 8, *pv_done = bars + 10, *p_full = bars + 12;   // a row tile each
    uint64_t *q_full = bars + 16, *drain = bars + 17;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 18);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    StepInfo *info = reinterpret_cast<StepInfo *>(bars + 20);
    // of each row: its multiplier; for either half of a step the greatest score; in the end the sums
    float *row_mult = reinterpret_cast<float *>(smem + F::ROW_OFF), *row_max = row_mult + 2 * kTile, *row_sum = row_max + 4 * kTile;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // ---- this CTA's rows and tokens (uniform) ----
    const int chunks = static_cast<int>(gridDim.x / static_cast<unsigned>(a.g.kv_heads));
    const int chunk = chunks - 1 - static_cast<int>(blockIdx.x / static_cast<unsigned>(a.g.kv_heads));   // longest first
    const int kvh = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.g.kv_heads));
    const SeqView sv = seq_view(a, blockIdx.z, blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0);
    const int all = sv.n * a.per_kv, first = chunk * 2 * kTile;
    if (first >= all) return;
    const int rows = all - first < 2 * kTile ? all - first : 2 * kTile;
    const int tiles = rows > kTile ? 2 : 1;
    int lo, hi;
    visible(a, sv, first / a.per_kv, (first + rows - 1) / a.per_kv, lo, hi);
    int begin = lo & ~(kTile - 1), steps = hi > lo ? (hi - begin + kTile - 1) / kTile : 0;
    int pieces = 1;
    if (a.splits > 1 && steps > 0) {                      // this piece's share of the steps
        const int per = max((steps + a.splits - 1) / a.splits, a.min_units);
        pieces = (steps + per - 1) / per;
        if (static_cast<int>(blockIdx.y) >= pieces) return;
        begin += static_cast<int>(blockIdx.y) * per * kTile;
        steps = min(per, steps - static_cast<int>(blockIdx.y) * per);
    } else if (blockIdx.y > 0) {
        return;
    }

    if (threadIdx.x == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&k_full[s], 4);
            mbar_init(&k_empty[s], 1);
            mbar_init(&v_full[s], 4);
            mbar_init(&v_empty[s], 1);
            mbar_init(&s_full[s], 1);
            mbar_init(&pv_done[s], 1);
            mbar_init(&p_full[s], 8);
        }
        mbar_init(q_full, 16);
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // the same answer for the whole warp, whose lanes go on together
    auto wait_warp = [&](uint64_t *bar, unsigned parity) {
        bool there = false;                               // (the clock is read only when it takes long)
        for (int n = 0; n < 16 && !there; ++n) there = mbar_try_wait(bar, parity);
        return __all_sync(0xffffffffu, there || mbar_wait_bounded(bar, parity, abort_flag)) != 0;
    };
    auto give_up = [&]() {
        *abort_flag = 1;
        set_error(a.err, ERR_TIMEOUT);
    };

    if (warp >= kMmaWarp) {
        if (warp == kMmaWarp && steps > 0) {
            const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0);
            const int row_tiles = __shfl_sync(0xffffffffu, tiles, 0);
            const uint32_t bar0 = smem_u32(bars);         // barriers as above, 8 bytes each
            const uint64_t q0 = smem_desc_k128(smem_u32(sq)), k0 = smem_desc_k128(smem_u32(sk)), v0 = smem_desc_k128(smem_u32(sv_));
            // S_i = Q_i K^T of step j (descriptors count 16-byte units)
            auto scores = [&](int i, int j) {
                constexpr uint32_t id = idesc_f16_f32(kTile, kTile);
                const uint64_t qa = q0 + i * (F::Q_BYTES / 16), kb = k0 + (j & 1) * (F::K_BYTES / 16);
                const uint32_t d = t0 + i * kTile;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss_one(d, qa + (k >> 2) * (kTile * 8) + 2 * (k & 3), kb + (k >> 2) * (kTile * 8) + 2 * (k & 3), id, k == 0 ? 0u : 1u);
                commit_one(bar0 + 8 * (8 + i));
            };
            // O_i += P_i V of step j
            auto values = [&](int i, int j) {
                constexpr uint32_t id = idesc_f16_f32(kTile, D);
                const uint64_t vb = v0 + (j & 1) * (F::V_BYTES / 16);
                const uint32_t pa = t0 + i * kTile, d = t0 + 2 * kTile + i * kTile;
                const uint32_t sum = j > 0 ? 1u : 0u;
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k)      // either half's P stands where its scores began
                    mma_ts_one(d, pa + (k >> 2) * kHalf + 8 * (k & 3), vb + (k >> 2) * (D * 8) + 2 * (k & 3), id, k == 0 ? sum : 1u);
            };
            bool ok = wait_warp(q_full, 0u) && wait_warp(&k_full[0], 0u);
            tc_fence_after();
            if (ok) {
                for (int i = 0; i < row_tiles; ++i) scores(i, 0);
                commit_one(smem_u32(&k_empty[0]));
            }
            for (int j = 0, more = 1; ok && more; ++j) {
                more = __shfl_sync(0xffffffffu, static_cast<volatile int &>(info[j % kInfos].step), 0) >= 0;
                ok = wait_warp(&v_full[j & 1], (j >> 1) & 1u);
                if (ok && more) ok = wait_warp(&k_full[(j + 1) & 1], ((j + 1) >> 1) & 1u);
                for (int i = 0; ok && i < row_tiles; ++i) {
                    ok = wait_warp(&p_full[i], j & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    values(i, j);
                    if (more) scores(i, j + 1);
                    else commit_one(bar0 + 8 * (10 + i));
                }
                if (ok) {                                 // step j's V and step j + 1's K have been multiplied
                    commit_one(smem_u32(&v_empty[j & 1]));
                    commit_one(smem_u32(&k_empty[(j + 1) & 1]));
                }
            }
            if (!ok && lane == 0) give_up();
            __syncwarp();
            commit_one(smem_u32(drain));                  // nothing of this CTA's is in flight when tensor memory is freed
            mbar_wait_bounded(drain, 0u, nullptr);
        }
    } else if (warp >= kKeyWarp) {
        const bool keys = warp < kValWarp;
        const int tid = threadIdx.x & (kTile - 1), w4 = warp & 3;
        // ---- codes to operands ----
        const int32_t *table = a.table + blockIdx.z * a.table_ld;
        const int page_mask = (1 << a.g.page_shift) - 1;
        const int64_t page_bytes = a.g.page_bytes;
        const uint8_t *mine = a.g.data + kvh * a.g.block_bytes;
        const uint32_t v_off = a.g.v_off, kg_off = a.g.kg_off, vg_off = a.g.vg_off;
        // tokens beyond the visible ones take the nearest visible one's place in memory; their grids are dropped
        auto near = [&](int tok) { return max(lo, min(tok, hi - 1)); };
        auto block_of = [&](int page, bool &out) {
            out = static_cast<uint32_t>(page) >= static_cast<uint64_t>(a.g.pages);
            return mine + (out ? 0 : page) * page_bytes;
        };
        // a power of two that brings the largest of the warp's scales to [1, 2); NaN and -0 (bad tokens) apart
        auto exponent = [&](int big) {
            big = __reduce_max_sync(0xffffffffu, big);
            const int e = static_cast<int>(static_cast<uint32_t>(big) >> 23) - 127;
            return big == 0 ? 0 : e < -100 ? -100 : e;
        };
        auto power = [](int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); };
        const __half2 sixteenth = __float2half2_rn(0.0625f);
        bool ok = true;
        if (keys && steps > 0) {
            uint32_t kw[4 * C], kg[NG];
            unsigned gone = 0u;                           // bits of the step in kw
            int page = 0;
            auto key_page = [&](int j) { page = table[near(begin + j * kTile + tid) >> a.g.page_shift]; };
            auto key_codes = [&](int j) {
                const int tok = begin + j * kTile + tid, at = near(tok) & page_mask;
                bool out;
                const uint8_t *blk = block_of(page, out);
                const unsigned votes = __ballot_sync(0xffffffffu, out);
                gone = (votes & 1u) | (votes >> 15 & 2u);
                if (votes && lane == 0) set_error(a.err, ERR_RANGE);
                const uint4 *pk = reinterpret_cast<const uint4 *>(blk + at * (D / 2));
#pragma unroll
                for (int i = 0; i < C; ++i) *reinterpret_cast<uint4 *>(&kw[4 * i]) = pk[i];
                const uint32_t *pg = reinterpret_cast<const uint32_t *>(blk + kg_off) + at * NG;
#pragma unroll
                for (int g = 0; g < NG; ++g) kg[g] = out || tok < lo || tok >= hi ? 0u : pg[g];
            };
            key_page(0);
            key_codes(0);
            if (steps > 1) key_page(1);
            for (int j = 0, n = 0; j < steps; ++n) {      // n: steps as they are taken
                const int s = n & 1;
                int big = 0;
#pragma unroll
                for (int g = 0; g < NG; ++g) big = max(big, kg[g] < 0x7F800000u ? static_cast<int>(kg[g]) : 0);
                const int kf = exponent(big) - kKeyRoom;
                const bool again = any_turning(false);
                ok = ok && wait_warp(&k_empty[s], ((n >> 1) & 1u) ^ 1u);   // (once it gave up it goes along without waiting)
                const float down = power(-kf);
                uint8_t *row = sk + s * F::K_BYTES + tid * 128;
                // the token's words stand as [t][w]: channels 32 w + 8 t .. + 7, one 16-byte chunk each
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float sc = __uint_as_float(kg[g] & 0xFFFF0000u) * down, z = __uint_as_float(kg[g] << 16);
                    const __half2 s2 = __float2half2_rn(sc), z2 = __float2half2_rn(z + 1024.0f), y2 = __float2half2_rn(-64.0f - z);
#pragma unroll
                    for (int w = g * GC; w < (g + 1) * GC; ++w)
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t x = kw[t * C + w], y = x >> 8;
                            uint32_t h[4] = {(x & 0x000f000fu) | 0x64006400u, (x & 0x00f000f0u) | 0x64006400u,
                                             (y & 0x000f000fu) | 0x64006400u, (y & 0x00f000f0u) | 0x64006400u};
                            __half2 *v = reinterpret_cast<__half2 *>(h);
                            v[0] = __hmul2(__hsub2(v[0], z2), s2);
                            v[1] = __hmul2(__hfma2(v[1], sixteenth, y2), s2);
                            v[2] = __hmul2(__hsub2(v[2], z2), s2);
                            v[3] = __hmul2(__hfma2(v[3], sixteenth, y2), s2);
                            const int ch = 4 * w + t;
                            *reinterpret_cast<uint4 *>(row + (ch >> 3) * (kTile * 128) + (((ch & 7) ^ (tid & 7)) << 4)) =
                                make_uint4(h[0], h[1], h[2], h[3]);
                        }
                }
                if (lane == 0) {
                    StepInfo &in = info[n % kInfos];
                    if (w4 == 0) in.step = !again && j + 1 == steps ? -1 - j : j;
                    in.key_up[w4] = power(kf);
                    in.gone[w4] = static_cast<uint8_t>(gone | (in.out[w4] ? 4u : 0u));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&k_full[s]);
                if (again) continue;                      // (where nothing is left over, with no token)
                ++j;
                if (j < steps) {
                    key_codes(j);
                    if (j + 1 < steps) key_page(j + 1);
                }
            }
        } else if (steps > 0) {
            constexpr int PER = (NG + 1) / 2;                 // lanes p and p + 16 have the pair of tokens p, each other groups
            const int pair = lane & 15;
            uint32_t vg0[PER], vg1[PER], next0[PER], next1[PER];   // grids of this step, of the next
            int vpage = 0;
            auto value_page = [&](int j) { vpage = table[near(begin + j * kTile + 32 * w4 + 2 * pair) >> a.g.page_shift]; };
            auto value_grids = [&](int j) {
                const int t2 = begin + j * kTile + 32 * w4 + 2 * pair;
                bool out;
                const uint32_t *p = reinterpret_cast<const uint32_t *>(block_of(vpage, out) + vg_off);
                const bool on0 = !out && t2 >= lo && t2 < hi, on1 = !out && t2 + 1 >= lo && t2 + 1 < hi;
    #pragma unroll
                for (int i = 0; i < PER; ++i) {
                    next0[i] = on0 ? p[(t2 & page_mask) * NG + group_of<NG>(i)] : 0u;
                    next1[i] = on1 ? p[((t2 + 1) & page_mask) * NG + group_of<NG>(i)] : 0u;
                }
            };
            auto take_grids = [&](int j) {                // step j's; those of the one after it are asked for
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    vg0[i] = next0[i];
                    vg1[i] = next1[i];
                }
                if (j + 1 < steps) value_grids(j + 1);
                if (j + 2 < steps) value_page(j + 2);
            };
            // Of the 32 tokens those `left` to take, in the end those left over; val_exp is E + kValRoom, biased.
            int val_exp = kLeastE;
            unsigned left = 0xffffffffu;
            auto fit = [&]() {
                uint32_t top = 0x80008000u;                   // greatest scales of the two as bf16 (a bad token's is below 0)
    #pragma unroll
                for (int i = 0; i < PER; ++i) top = __vmaxs2(top, __byte_perm(vg0[i], vg1[i], 0x7632));
                if constexpr (NG > 1) top = __vmaxs2(top, __shfl_xor_sync(0xffffffffu, top, 16));
                unsigned out = 0u;
                if (left != 0xffffffffu || __any_sync(0xffffffffu, misfit(static_cast<int>(top >> 7 & 0xffu), val_exp) || misfit(static_cast<int>(top >> 23 & 0xffu), val_exp))) {
                    const int b = static_cast<int>(__shfl_sync(0xffffffffu, top, lane >> 1) >> (lane & 1 ? 23 : 7) & 0xffu);
                    const unsigned over = left == 0u ? 0u : refit_tokens(b, left, val_exp);
                    out = ~left | over;
                    left = over;
                } else {
                    left = 0u;
                }
                return out;
            };
            const int vr = lane >> 2, vb = lane & 3;      // channels 4 vr .. + 3 of each chunk, 8-token block vb of the warp's 32
            uint2 *pairs = reinterpret_cast<uint2 *>(spairs) + w4 * 16 * NG;   // [group][pair]
            uint32_t vw[4 * C];
            int page = 0;
            auto block_at = [&](int j) { return max(lo & ~7, min(begin + j * kTile + 32 * w4 + 8 * vb, (hi - 1) & ~7)); };
            auto code_page = [&](int j) { page = table[block_at(j) >> a.g.page_shift]; };
            auto codes = [&](int j) {
                bool out;
                const uint4 *pv = reinterpret_cast<const uint4 *>(block_of(page, out) + v_off + (block_at(j) & page_mask) * (D / 2) + vr * 16 * C);
#pragma unroll
                for (int i = 0; i < C; ++i) *reinterpret_cast<uint4 *>(&vw[4 * i]) = pv[i];
            };
            code_page(0);
            value_page(0);
            codes(0);
            value_grids(0);
            if (steps > 1) {
                code_page(1);
                value_page(1);
            }
            take_grids(0);
            const __half2 m960 = __float2half2_rn(960.0f);
            // What step n takes is found, and the warps that turn keys told, before step n - 1 is turned, for which this
            // warp has to wait longer.
            unsigned out = 0u;
            bool again = false;
            auto look_at = [&](int n) {
                out = fit();
                if (lane == 0) {
                    StepInfo &in = info[n % kInfos];
                    in.out[w4] = out;
                    in.val_exp[w4] = static_cast<float>(val_exp - 127 - kValRoom);
                    in.val_down[w4] = power(127 + kValRoom - val_exp);
                }
                again = any_turning(left != 0u);
            };
            look_at(0);
            for (int j = 0, n = 0; j < steps; ++n) {
                const int s = n & 1;
                // scales and zero points of pairs of tokens, turned once by the warp
                const float down = power(127 + kValRoom - val_exp);
                out >>= 2 * pair;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const __half2 s2 = __floats2half2_rn(out & 1u ? 0.0f : __uint_as_float(vg0[i] & 0xFFFF0000u) * down,
                                                         out & 2u ? 0.0f : __uint_as_float(vg1[i] & 0xFFFF0000u) * down);
                    const __half2 z2 = __floats2half2_rn(__uint_as_float(vg0[i] << 16) + 1024.0f, __uint_as_float(vg1[i] << 16) + 1024.0f);
                    if (NG % 2 == 0 || 2 * i + (lane >> 4) < NG)
                        pairs[group_of<NG>(i) * 16 + pair] = make_uint2(*reinterpret_cast<const uint32_t *>(&s2), *reinterpret_cast<const uint32_t *>(&z2));
                }
                __syncwarp();
                const bool done = !again;
                if (done && j + 1 < steps) {
                    left = 0xffffffffu;
                    take_grids(j + 1);
                }
                if (!done || j + 1 < steps) look_at(n + 1);
                ok = ok && wait_warp(&v_empty[s], ((n >> 1) & 1u) ^ 1u);
                uint8_t *base = sv_ + s * F::V_BYTES + (w4 >> 1) * (D * 128);
                const int ch = 4 * (w4 & 1) + vb;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    __half2 s2[4], z2[4], y2[4];
                    {
                        const uint4 q0 = *reinterpret_cast<const uint4 *>(&pairs[g * 16 + 4 * vb]), q1 = *reinterpret_cast<const uint4 *>(&pairs[g * 16 + 4 * vb + 2]);
                        s2[0] = *reinterpret_cast<const __half2 *>(&q0.x);
                        z2[0] = *reinterpret_cast<const __half2 *>(&q0.y);
                        s2[1] = *reinterpret_cast<const __half2 *>(&q0.z);
                        z2[1] = *reinterpret_cast<const __half2 *>(&q0.w);
                        s2[2] = *reinterpret_cast<const __half2 *>(&q1.x);
                        z2[2] = *reinterpret_cast<const __half2 *>(&q1.y);
                        s2[3] = *reinterpret_cast<const __half2 *>(&q1.z);
                        z2[3] = *reinterpret_cast<const __half2 *>(&q1.w);
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) y2[t] = __hsub2(m960, z2[t]);     // -(64 + z)
#pragma unroll
                    for (int w = g * GC; w < (g + 1) * GC; ++w) {
                        uint32_t h[4][4];                 // [channel][pair of tokens]
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t x = vw[t * C + w], y = x >> 8;
                            h[0][t] = (x & 0x000f000fu) | 0x64006400u;
                            h[1][t] = (x & 0x00f000f0u) | 0x64006400u;
                            h[2][t] = (y & 0x000f000fu) | 0x64006400u;
                            h[3][t] = (y & 0x00f000f0u) | 0x64006400u;
                            __half2 *v0 = reinterpret_cast<__half2 *>(&h[0][t]), *v1 = reinterpret_cast<__half2 *>(&h[1][t]);
                            __half2 *v2 = reinterpret_cast<__half2 *>(&h[2][t]), *v3 = reinterpret_cast<__half2 *>(&h[3][t]);
                            *v0 = __hmul2(__hsub2(*v0, z2[t]), s2[t]);
                            *v1 = __hmul2(__hfma2(*v1, sixteenth, y2[t]), s2[t]);
                            *v2 = __hmul2(__hsub2(*v2, z2[t]), s2[t]);
                            *v3 = __hmul2(__hfma2(*v3, sixteenth, y2[t]), s2[t]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int d = 32 * w + 4 * vr + i;
                            *reinterpret_cast<uint4 *>(base + d * 128 + ((ch ^ (d & 7)) << 4)) = make_uint4(h[i][0], h[i][1], h[i][2], h[i][3]);
                        }
                    }
                }
                fence_async_smem();
                __syncwarp();                             // also: the pairs are read before the next step's are written
                if (lane == 0) mbar_arrive(&v_full[s]);
                if (!done) continue;
                ++j;
                if (j < steps) {
                    codes(j);
                    if (j + 1 < steps) code_page(j + 1);
                }
            }
        }
        if (!ok && lane == 0) give_up();
    } else {
        // ---- softmax: a thread a row and half of the step's tokens ----
        const int grp = warp >> 3, i = (warp >> 2) & 1, quad = warp & 3, tid = threadIdx.x & (kTile - 1);
        const int p = i * kTile + tid;
        const bool on = p < rows;
        const unsigned pr = first + (on ? p : 0), qi = pr / static_cast<unsigned>(a.per_kv);
        const int head = kvh * a.per_kv + static_cast<int>(pr - qi * a.per_kv);
        int see_lo, see_hi;
        visible(a, sv, qi, qi, see_lo, see_hi);
        const int all_lo = __reduce_max_sync(0xffffffffu, see_lo), all_hi = __reduce_min_sync(0xffffffffu, see_hi);
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16) + i * kTile, to = lanes + 2 * kTile;
        bool ok = true;                                   // no wait gave up
        // Q: the warp's 32 rows, LR lanes to a row, scaled into fp16 by a power of two of the row
        constexpr int LR = D <= 64 ? 8 : 16, RI = 32 / LR;
        const int64_t q_at = (sv.row0 + qi) * a.q_row + head * a.q_head;
        if (i < tiles && steps > 0) {
            const int sub = lane / LR, c = lane % LR;     // row of the RI at once, 16-byte chunk of the row
            constexpr int HR = LR / 2;                    // each group brings half of the rows
            uint4 raw[HR];
#pragma unroll
            for (int k = 0; k < HR; ++k) {
                const int r = grp * HR + k;
                const int64_t at = __shfl_sync(0xffffffffu, q_at, r * RI + sub);
                const bool mine = i * kTile + quad * 32 + r * RI + sub < rows && 8 * c < a.g.dim;
                const uint16_t *from = reinterpret_cast<const uint16_t *>(a.Q) + at + 8 * c;
                raw[k] = make_uint4(0u, 0u, 0u, 0u);
                if (mine && a.q_vec) raw[k] = *reinterpret_cast<const uint4 *>(from);
                else if (mine)
                    raw[k] = make_uint4(from[0] | from[1] << 16, from[2] | from[3] << 16, from[4] | from[5] << 16, from[6] | from[7] << 16);
            }
            uint8_t *tile = sq + i * F::Q_BYTES + (c >> 3) * (kTile * 128);
#pragma unroll
            for (int k = 0; k < HR; ++k) {
                const int row = quad * 32 + (grp * HR + k) * RI + sub;
                // the largest magnitude: 16-bit floats without their signs are ordered as integers
                uint32_t big = __vmaxu2(__vmaxu2(raw[k].x & 0x7fff7fffu, raw[k].y & 0x7fff7fffu), __vmaxu2(raw[k].z & 0x7fff7fffu, raw[k].w & 0x7fff7fffu));
#pragma unroll
                for (int o = 1; o < LR; o <<= 1) big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, o));
                const uint32_t most = max(big & 0xffffu, big >> 16);
                float down, up;
                q_powers(a.half ? __half2float(__ushort_as_half(static_cast<unsigned short>(most))) : __uint_as_float(most << 16), down, up);
                if (c == 0) row_mult[i * kTile + row] = up * a.scale2;
                auto scaled = [&](uint32_t w) {
                    float x, y;
                    if (a.half) {
                        const __half2 h = *reinterpret_cast<const __half2 *>(&w);
                        x = __low2float(h);
                        y = __high2float(h);
                    } else {
                        x = __uint_as_float(w << 16);
                        y = __uint_as_float(w & 0xffff0000u);
                    }
                    return pack_f16(x * down, y * down);
                };
                if (8 * c < F::DQ)
                    *reinterpret_cast<uint4 *>(tile + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
                        make_uint4(scaled(raw[k].x), scaled(raw[k].y), scaled(raw[k].z), scaled(raw[k].w));
            }
            fence_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
        float m = kFloor, l = 0.0f, mult = 0.0f;
        for (int j = 0, more = steps > 0; i < tiles && more; ++j) {
            ok = wait_warp(&s_full[i], j & 1u);           // and the products of the step before have been taken
            if (!ok && lane == 0) *abort_flag = 1;
            tc_fence_after();
            // (these products have read Q and K, so what came with them is there)
            if (j == 0) mult = row_mult[p];
            const StepInfo &in = info[j % kInfos];
            more = in.step >= 0;
            const int c0 = 2 * grp, j0 = begin + (more ? in.step : -1 - in.step) * kTile + grp * kHalf;
            const unsigned gone = *reinterpret_cast<const uint16_t *>(&in.gone[c0]);
            const uint32_t ts = lanes + grp * kHalf;
            const bool edge = gone != 0u || j0 < all_lo || j0 + kHalf > all_hi;
            // what scores of 32 tokens are multiplied with: never 0, as masked ones are -inf by then (all-zero rows and
            // keys, or a tiny caller's scale, come to 2^-229 and less), never infinite, as some may be 0; a score that
            // 2^-126 instead of less makes differ is below 2^-80 either way
            auto factor = [&](int c) { return fminf(fmaxf(mult * in.key_up[c0 + c], 1.17549435e-38f), 1.70141183e38f); };
            // the scores of the half's tokens 32 c .. + 31
            auto fetch = [&](int c, float (&v)[32]) {
                tmem_ld_32x32b_x32(ts + 32 * c, v);
                if (edge) {
                    asm volatile("" ::: "memory");        // a branch around this, not selects in every step
                    // bit e: the row sees token e of the 32
                    const int t0 = j0 + 32 * c, from = max(see_lo - t0, 0), upto = min(see_hi - t0, 32);
                    unsigned bits = (from < 32 ? 0xffffffffu << from : 0u) & ~in.out[c0 + c];
                    bits &= upto > 0 ? 0xffffffffu >> (32 - upto) : 0u;
                    if ((gone >> (8 * c)) & 1u) bits &= 0xffff0000u;
                    if ((gone >> (8 * c)) & 2u) bits &= 0x0000ffffu;
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((bits >> e) & 1u)) v[e] = -CUDART_INF_F;
                }
            };
            auto highest = [&](int c, const float (&v)[32]) {
                float x[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = fmaxf(v[q], v[q + 4]);
#pragma unroll
                for (int e = 8; e < 32; e += 8)
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[q] = fmaxf(x[q], fmaxf(v[e + q], v[e + q + 4]));
                return fmaf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), factor(c), in.val_exp[c0 + c]);
            };
            // exponentials at the maximum so far, packed
            auto powers = [&](int c, float (&v)[32], uint32_t *h) {
                const uint64_t k = twice(factor(c)), b = twice(in.val_exp[c0 + c] - m);
                uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    fma2(v[e], v[e + 1], k, b);
                    v[e] = ex2(v[e]);
                    v[e + 1] = ex2(v[e + 1]);
                    add2(sum[(e >> 1) & 3], v[e], v[e + 1]);
                    h[e >> 1] = pack_f16(v[e], v[e + 1]);
                }
                return total(sum) * in.val_down[c0 + c];
            };
            const int pair_bar = 1 + 4 * i + quad;        // this warp and the other group's warp of these rows
            bool raise = j == 0;
            if (j > 0) {
                // taken at the old maximum at once; only where one exceeds 2^(kAbove + kRaise) (seldom) it is all done again
                uint32_t h[32];
                float v[32];
                fetch(0, v);
                float sum = powers(0, v, h);
                fetch(1, v);
                sum += powers(1, v, h + 16);
                __half2 x[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = __hmax2(as_half2(h[q]), as_half2(h[q + 4]));
#pragma unroll
                for (int e = 8; e < 32; e += 4)
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[q] = __hmax2(x[q], as_half2(h[e + q]));
                x[0] = __hmax2(__hmax2(x[0], x[1]), __hmax2(x[2], x[3]));
                raise = any_of_64(pair_bar, !ok || __hgt(__hmax(__low2half(x[0]), __high2half(x[0])), __float2half(32768.0f)));
                if (!raise) {
                    tmem_st_x32(ts, h);
                    l += sum;
                }
            }
            if (raise) {
                asm volatile("" ::: "memory");
                float top = kFloor;
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    float v[32];
                    fetch(c, v);
                    top = fmaxf(top, highest(c, v) - kAbove);
                }
                // the other half's, from the other group
                row_max[grp * 2 * kTile + p] = ok ? top : CUDART_NAN_F;
                sync_64(pair_bar);
                const float theirs = row_max[(1 - grp) * 2 * kTile + p];
                ok = ok && theirs == theirs;
                if (!ok) break;                           // one of the two gave up: both leave at the same barrier
                top = fmaxf(top, theirs);
                const float now = fmaxf(m, top), f = ex2(m - now);
                m = now;
                l *= f;
                if (j > 0) {                              // either group has half of the channels
#pragma unroll 1
                    for (int c = grp * (D / 32); c < (grp + 1) * (D / 32); ++c) {
                        float o[16];
                        tmem_ld_x16(to + 16 * c, o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] *= f;
                        tmem_st_x16(to + 16 * c, o);
                    }
                }
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    float v[32];
                    uint32_t h[16];
                    fetch(c, v);
                    l += powers(c, v, h);
                    tmem_st_x16(ts + 16 * c, h);          // in place of scores that have been read
                }
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[i]);
        }
        if (i < tiles) {
            row_sum[grp * 2 * kTile + p] = l;
            asm volatile("bar.sync %0, 256;" ::"r"(9 + i) : "memory");
            l += row_sum[(1 - grp) * 2 * kTile + p];
            if (steps > 0) {
                ok = ok && wait_warp(&pv_done[i], 0u);
                tc_fence_after();
                if (!ok && lane == 0) give_up();
            }
        }
        if (i < tiles) {
            float *slot = a.part + (static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x) * a.splits * (2 * kTile * (D + 2)) +
                          static_cast<int64_t>(blockIdx.y) * (2 * kTile * (D + 2));
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // a row that sees nothing is zero; NaN stays
            // whole rows go through shared memory (every product has been taken, Q's place is free) and out
            // LR lanes to a row: a thread's own row would be 8 to 16 bytes a line in each store
            uint8_t *stage = sq + i * F::Q_BYTES + quad * 32 * (F::DQ * 2);
#pragma unroll 1
            for (int c = grp; c < D / 32; c += 2) {
                float v[32];
                if (steps > 0) {
                    tmem_ld_32x32b_x32(to + 32 * c, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0.0f;
                }
                if (pieces > 1) {
                    if (on)
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<float4 *>(slot + p * D + 32 * c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float x = v[e + 2 * k] * inv, y = v[e + 2 * k + 1] * inv;
                            w[k] = a.half ? pack_f16(x, y) : pack_bf16(x, y);
                        }
                        *reinterpret_cast<uint4 *>(stage + lane * (F::DQ * 2) + (((4 * c + e / 8) ^ (lane & (LR - 1))) << 4)) =
                            make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (pieces == 1) {
                if (on && a.lse && grp == 0)
                    a.lse[(sv.row0 + qi) * a.q_heads + head] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * 0.693147180559945309f;
                asm volatile("bar.sync %0, 256;" ::"r"(9 + i) : "memory");
                const int64_t o_at = (sv.row0 + qi) * a.o_row + head * a.o_head;
                const int sub = lane / LR, c = lane % LR;
#pragma unroll 4
                for (int r = grp * (LR / 2); r < (grp + 1) * (LR / 2); ++r) {
                    const int row = r * RI + sub;
                    const int64_t at = __shfl_sync(0xffffffffu, o_at, row);
                    if (i * kTile + quad * 32 + row >= rows || 8 * c >= a.g.dim) continue;
                    const uint4 w = *reinterpret_cast<const uint4 *>(stage + row * (F::DQ * 2) + ((c ^ (row & (LR - 1))) << 4));
                    uint16_t *dst = reinterpret_cast<uint16_t *>(a.out) + at + 8 * c;
                    if (a.o_vec) {
                        *reinterpret_cast<uint4 *>(dst) = w;
                    } else {
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int k = 0; k < 8; ++k) dst[k] = static_cast<uint16_t>(u[k >> 1] >> (16 * (k & 1)));
                    }
                }
            }
            if (on && pieces > 1 && grp == 0) {
                slot[2 * kTile * D + p] = m;
                slot[2 * kTile * (D + 1) + p] = l;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// Joins the pieces of an item: the block of item x and sequence y, 8 rows a pass.
__global__ void __launch_bounds__(256) k_attend_join_tiles(const AttendArgs a) {
    const int chunks = static_cast<int>(gridDim.x / static_cast<unsigned>(a.g.kv_heads));
    const int chunk = chunks - 1 - static_cast<int>(blockIdx.x / static_cast<unsigned>(a.g.kv_heads));
    const int kvh = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.g.kv_heads));
    const SeqView sv = seq_view(a, blockIdx.z, false);
    const int all = sv.n * a.per_kv, first = chunk * 2 * kTile;
    int pieces = 0, rows = 0;
    if (first < all) {
        rows = all - first < 2 * kTile ? all - first : 2 * kTile;
        int lo, hi;
        visible(a, sv, first / a.per_kv, (first + rows - 1) / a.per_kv, lo, hi);
        const int steps = hi > lo ? (hi - (lo & ~(kTile - 1)) + kTile - 1) / kTile : 0;
        const int per = max((steps + a.splits - 1) / a.splits, a.min_units);
        pieces = (steps + per - 1) / per;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (pieces <= 1) return;
    const int D = a.g.D, quads = D / 4;
    const int64_t size = 2 * kTile * (D + 2);
    const float *base = a.part + (static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x) * a.splits * size;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < rows * quads; i += gridDim.y * 256) {
        const int row = i / quads, d = 4 * (i % quads);
        if (d >= a.g.dim) continue;
        float big = kFloor, sum = 0.0f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < pieces; ++s) big = fmaxf(big, base[s * size + 2 * kTile * D + row]);
        for (int s = 0; s < pieces; ++s) {
            const float *p = base + s * size;
            const float f = ex2(p[2 * kTile * D + row] - big);
            const float4 u = *reinterpret_cast<const float4 *>(p + row * D + d);
            sum = fmaf(f, p[2 * kTile * (D + 1) + row], sum);
            v = make_float4(fmaf(f, u.x, v.x), fmaf(f, u.y, v.y), fmaf(f, u.z, v.z), fmaf(f, u.w, v.w));
        }
        const unsigned pr = first + row, q = pr / static_cast<unsigned>(a.per_kv);
        finish(a, sv.row0 + q, kvh * a.per_kv + static_cast<int>(pr - q * a.per_kv), d, v, big, sum);
    }
}

template <int C, int GC>
cudaError_t launch_tiles(const AttendArgs &a, const dim3 &grid, cudaStream_t s) {
    using F = TcCfg<C, GC>;
    static std::atomic<uint64_t> raised{0};
    const cudaError_t e = raise_smem(reinterpret_cast<const void *>(k_attend_tiles<C, GC>), F::SMEM_ASKED, raised);
    if (e != cudaSuccess) return e;
    k_attend_tiles<C, GC><<<grid, kThreads, F::SMEM_ASKED, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_tiles(const AttendArgs &a, cudaStream_t s) {
    const int C = a.g.D / 32, GC = C / a.g.groups;
    const unsigned items = static_cast<unsigned>(ceil_div(a.max_q * a.per_kv, 2 * kTile) * a.g.kv_heads);
    const dim3 grid(items, static_cast<unsigned>(a.splits), static_cast<unsigned>(a.seqs));
    cudaError_t e;
    if (C == 2) e = GC == 1 ? launch_tiles<2, 1>(a, grid, s) : launch_tiles<2, 2>(a, grid, s);
    else if (C == 3) e = launch_tiles<3, 1>(a, grid, s);
    else if (GC == 1) e = launch_tiles<4, 1>(a, grid, s);
    else if (GC == 2) e = launch_tiles<4, 2>(a, grid, s);
    else e = launch_tiles<4, 4>(a, grid, s);
    if (e != cudaSuccess || a.splits == 1) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(items, 8, static_cast<unsigned>(a.seqs));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_attend_join_tiles, a);
}

}  // namespace qe
