// What both attention kernels over the 4-bit cache share on the device: loading query
// rows, and finishing output rows.
#pragma once

#include <cuda_fp16.h>
#include <math_constants.h>

#include "qe_attend.h"

namespace qe {

constexpr float kRaise = 8.0f;            // log2 of how far a score may exceed the running maximum
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

// Four channels of a finished row, from the unnormalised sums relative to the maximum `m` (log2 units).
__device__ __forceinline__ void finish(const AttendArgs &a, int64_t row, int head, int d, const float4 &v, float m, float l) {
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
