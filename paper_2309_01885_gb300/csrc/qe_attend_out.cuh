// What both attention kernels over the 4-bit cache share on the device: loading query
// rows, and finishing output rows.
#pragma once

#include <cuda_fp16.h>
#include <math_constants.h>

#include "qe_attend.h"

namespace qe {

constexpr float kRaise = 8.0f;            // log2 of how far a score may exceed the running maximum
constexpr float kAbove = 7.0f;            // probabilities are taken 2^7 above it, up to 2^15: fp16's range begins lower for them

// fp16 holds a step's value scales relative to a power of two of their channel group, 2^e_g: within 2^-kWindow and 2 of it.
// The largest of these, 2^e, P takes over: the running maximum is then one of score + e, of what a token adds to the
// result.  A token with a scale that does not fit is added by itself, in binary32.  Exponents are biased as in binary32.
constexpr int kWindow = 7, kHeadroom = 2;
constexpr int kMostExp = 127 + 40, kLeastExp = 127 - 40;   // of e: a change of it multiplies the sum of P, which stays finite
constexpr int kMostApart = 30;            // how far an e_g is below e at most, likewise

__device__ __forceinline__ int scale_exp(uint32_t grid) { return static_cast<int>(grid >> 23 & 0xffu); }
__device__ __forceinline__ float power(int biased) { return __uint_as_float(static_cast<uint32_t>(biased) << 23); }

// Not 0 where one of two scales in fp16 is outside [2^-kWindow, 2): these are the ones whose upper three bits are 001.
__device__ __forceinline__ uint32_t misfits(uint32_t s2) { return (s2 ^ 0x20002000u) & 0xE000E000u; }

// Whether a scale's exponent does not fit e_g (0, 1: unseen, all zeros, at the least or marked bad; no matter).
__device__ __forceinline__ bool unfit(int b, int eg) { return b > 1 && static_cast<unsigned>(b - (eg - kWindow)) > kWindow; }

// The channel groups of lanes that share a step's value grids out: lanes p and p + 16 have the pair of tokens p.
template <int NG>
__device__ __forceinline__ int group_of(int i) { return NG == 1 ? 0 : min(2 * i + static_cast<int>(threadIdx.x >> 4 & 1u), NG - 1); }

// For 32 tokens, not all of which fit: new e and e_g (of the lane's groups), such that of each group at least a quarter
// of its tokens fit, and the tokens of which a group does not (bits p and p + 16: tokens 2 p and 2 p + 1).  t0, t1: the
// exponent that P takes over of either token where it is added by itself: its largest scale's, at most e.
template <int PER>
__device__ __forceinline__ unsigned refit(const uint32_t (&v0)[PER], const uint32_t (&v1)[PER], int &e, int (&eg)[PER], int &t0, int &t1) {
    const int half = threadIdx.x & 16;                    // this lane's groups: bits 0 .. 15 or 16 .. 31 of a vote
    auto votes = [&](bool x) { return __ballot_sync(0xffffffffu, x) >> half & 0xffffu; };
    auto greatest = [&](int x) {
        const int a = __reduce_max_sync(0xffffffffu, half ? 0 : x), b = __reduce_max_sync(0xffffffffu, half ? x : 0);
        return half ? b : a;
    };
    t0 = t1 = e = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b0 = scale_exp(v0[i]), b1 = scale_exp(v1[i]), most = greatest(max(b0, b1));
        if (most > 1) eg[i] = most + kHeadroom;           // (an empty group keeps its e_g)
        if (__any_sync(0xffffffffu, unfit(b0, eg[i]) || unfit(b1, eg[i]))) {
            bool left0 = b0 > 1, left1 = b1 > 1, done = most <= 1;
            const int n = __popc(votes(left0)) + __popc(votes(left1));
            while (__any_sync(0xffffffffu, !done)) {
                const int top = greatest(max(left0 ? b0 : 0, left1 ? b1 : 0));
                const bool in0 = left0 && b0 >= top - (kWindow - kHeadroom), in1 = left1 && b1 >= top - (kWindow - kHeadroom);
                left0 = left0 && !in0;
                left1 = left1 && !in1;
                const int fit = __popc(votes(in0)) + __popc(votes(in1));
                const bool last = (votes(left0) | votes(left1)) == 0u;
                if (!done) {
                    eg[i] = top + kHeadroom;
                    done = 4 * fit >= n || last;
                }
            }
        }
        e = max(e, eg[i]);
        t0 = max(t0, b0);
        t1 = max(t1, b1);
    }
    e = min(max(__reduce_max_sync(0xffffffffu, e), kLeastExp), kMostExp);
    bool out0 = false, out1 = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        eg[i] = min(max(eg[i], max(e - kMostApart, kLeastExp)), e);
        out0 = out0 || unfit(scale_exp(v0[i]), eg[i]);
        out1 = out1 || unfit(scale_exp(v1[i]), eg[i]);
    }
    if (!__any_sync(0xffffffffu, out0 || out1)) return 0u;
    t0 = max(t0, __shfl_xor_sync(0xffffffffu, t0, 16));
    t1 = max(t1, __shfl_xor_sync(0xffffffffu, t1, 16));
    t0 = max(min(t0, e), e - 80);
    t1 = max(min(t1, e), e - 80);
    const unsigned all0 = __ballot_sync(0xffffffffu, out0), all1 = __ballot_sync(0xffffffffu, out1);
    return ((all0 | all0 >> 16) & 0xffffu) | (all1 | all1 >> 16) << 16;
}

constexpr float kFloor = -1.0e30f;        // the running maximum before the first visible score

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
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


// down = 2^-e and up = 2^e with big 2^-e in [2^14, 2^15): a query row scaled into fp16's
// range (zeros and subnormals keep a finite factor; an infinity or NaN stays one).
__device__ __forceinline__ void q_powers(float big, float &down, float &up) {
    int e = static_cast<int>(__float_as_uint(big) >> 23) - 127 - 14;
    if (e < -126) e = -126;
    if (e > 113) e = 113;
    down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

// The next kernel in the stream may begin, if it was launched so; and waiting for the last one's end and its writes.
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Where the first pass keeps a row's head: sums, and the offsets of maxima and totals behind all of them.
struct First {
    float *sums, *most, *total;
};

__device__ __forceinline__ First first_of(const AttendArgs &a, int64_t row, int head) {
    const int64_t all = a.rows * a.q_heads, at = row * a.q_heads + head;
    float *stats = a.first + all * a.g.D;
    return First{a.first + at * a.g.D, stats + at, stats + all + at};
}

// Four channels of a finished row of the sequence, from the unnormalised sums relative to the maximum `m` (log2 units).
__device__ __forceinline__ void finish(const AttendArgs &a, const SeqView &sv, int64_t row, int head, int d, float4 v, float m, float l) {
    if (a.first_pass) {
        const First f = first_of(a, row, head);
        *reinterpret_cast<float4 *>(f.sums + d) = v;
        if (d == 0) {
            *f.most = m;
            *f.total = l;
        }
        return;
    }
    if (sv.from > 0) {                                    // what the prefix adds
        const First f = first_of(a, row, head);
        const float4 u = *reinterpret_cast<const float4 *>(f.sums + d);
        const float most = *f.most, top = fmaxf(m, most), mine = ex2(m - top), its = ex2(most - top);
        v = make_float4(fmaf(its, u.x, mine * v.x), fmaf(its, u.y, mine * v.y), fmaf(its, u.z, mine * v.z), fmaf(its, u.w, mine * v.w));
        l = fmaf(its, *f.total, mine * l);
        m = top;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;       // a row that sees nothing is zero; NaN stays
    uint16_t *to = reinterpret_cast<uint16_t *>(a.out) + row * a.o_row + head * a.o_head + d;
    uint2 w;
    if (a.half) {
        w.x = pack_f16(v.x * inv, v.y * inv);
        w.y = pack_f16(v.z * inv, v.w * inv);
    } else {
        w.x = pack_bf16(v.x * inv, v.y * inv);
        w.y = pack_bf16(v.z * inv, v.w * inv);
    }
    if (a.o_vec) {
        *reinterpret_cast<uint2 *>(to) = w;
    } else {
        to[0] = static_cast<uint16_t>(w.x);
        to[1] = static_cast<uint16_t>(w.x >> 16);
        to[2] = static_cast<uint16_t>(w.y);
        to[3] = static_cast<uint16_t>(w.y >> 16);
    }
    if (d == 0 && a.lse)
        a.lse[row * a.q_heads + head] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * 0.693147180559945309f;
}

}  // namespace qe
