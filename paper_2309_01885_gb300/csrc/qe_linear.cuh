// A quantized layer as products take it: the layout of its bytes, and turning codes into
// matrix operands.
//
// Codes come in units of 16 rows x 64 columns, a row tile's units one after the other, so
// that whoever walks along a row tile reads one stream.  A unit has B words for each of 32
// lanes (B bits a code: 2, 3, 4 or 8).  Lane 4 r + t holds rows r and r + 8 (half h = 0, 1),
// of either 32-column chunk c = 0, 1 four pairs p of neighbouring columns, 32 c + 8 p + 2 t and
// the next, each in the low bits of a word's two halves once shifted: so the m16n8k16 operand
// wants them, and so a 16 x 128-bit store of tensor memory takes them.
//   B = 2  word c, bits 2 (4 h + p);   B = 4  word 2 c + h, bits 4 p;
//   B = 8  word 4 c + 2 h + p / 2, bits 8 (p mod 2);
//   B = 3  pairs i = 8 c + 4 h + p: word i / 5, bits 3 (i mod 5); i = 15 takes the bit that each
//          half has left over, bit j of its code in word j: 32 codes in 96 bits.
// (Bits are those of the pair's first column; its second column's are 16 above.)
// Behind the codes lie scales (fp32), 16 to a row tile and group, and zeros (one byte): a word for
// each pair of row tiles, group and r holds those of rows r and r + 8 of the first and of the second.
//
// c - z is exact in both 16-bit types.  A code below the leading bit of 2^7 (bf16) or 2^10
// (fp16) makes 2^7 + c 2^s by or-ing alone; one fused multiply-add takes s and the zero out.
#pragma once

#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "../../include/qe.h"
#include "qe_common.cuh"

namespace qe {

constexpr int kUnitCols = 64, kTileRows = 16;

// Units that the matrix units' accumulators add up before their sums go to registers (or shared memory): 8192 columns (up to
// twice as many where a CTA of the few-rows kernel has no more).  They lose up to a unit in the last place with each addition,
// of 16 columns, always towards zero: 512 of them make 2^-14 of a sum of one sign at most (measured: a tenth of that), which 16
// bits do not show; those of 2^20 columns, shared by eight CTAs, 2^-10, more than fp16's rounding.
constexpr int kSegmentUnits = 128;

struct LinearGeom {
    const uint8_t *codes;
    const float *scales;
    const uint32_t *zeros;
    int64_t q, p;
    int bits;                 // as stored: 2, 3, 4 or 8
    int units;                // of a row tile
    int row_tiles;
    int groups, group_units;  // grids of a row; units that share one
};

struct LinearArgs {
    LinearGeom g;
    const void *x;
    int64_t ldx, rows;
    int half;                 // fp16, else bf16
    int x_vec;                // 16-byte loads of x are aligned
    const void *bias;
    int bias_dtype;
    int act;
    const void *residual;
    int64_t ldr;
    void *y;
    int64_t ldy;
    unsigned *err;
};

__host__ __device__ constexpr int stored_bits(int bits) { return bits <= 4 ? bits : 8; }

// Place among a unit's words of a lane's word j of B.
__host__ __device__ constexpr int unit_word(int B, int lane, int j) {
    return B == 3 ? 32 * j + lane : B == 8 ? 128 * (j >> 2) + 4 * lane + (j & 3) : B * lane + j;
}

// A lane's words of a unit; `from` is the lane's own place in it.
template <int B>
__device__ __forceinline__ void load_unit(const uint8_t *from, uint32_t (&w)[B]) {
    if constexpr (B == 3) {
#pragma unroll
        for (int j = 0; j < 3; ++j) asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[j]) : "l"(from + 128 * j));
    } else if constexpr (B == 2) {
        asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(from));
    } else {
#pragma unroll
        for (int j = 0; j < B; j += 4)
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[j]), "=r"(w[j + 1]), "=r"(w[j + 2]), "=r"(w[j + 3])
                         : "l"(from + 128 * j));
    }
}

// The same from shared memory.
template <int B>
__device__ __forceinline__ void read_unit(const uint8_t *unit, int lane, uint32_t (&w)[B]) {
    if constexpr (B == 3) {
#pragma unroll
        for (int j = 0; j < 3; ++j) w[j] = reinterpret_cast<const uint32_t *>(unit)[32 * j + lane];
    } else if constexpr (B == 2) {
        const uint2 v = reinterpret_cast<const uint2 *>(unit)[lane];
        w[0] = v.x;
        w[1] = v.y;
    } else {
#pragma unroll
        for (int j = 0; j < B; j += 4) {
            const uint4 v = reinterpret_cast<const uint4 *>(unit + 128 * j)[lane];
            w[j] = v.x;
            w[j + 1] = v.y;
            w[j + 2] = v.z;
            w[j + 3] = v.w;
        }
    }
}

// Pairs of 16-bit floats as words.
template <bool HALF>
struct Pairs {
    static constexpr int kBase = HALF ? 1024 : 128;
    static constexpr uint32_t kLead = HALF ? 0x64006400u : 0x43004300u;
    static __device__ __forceinline__ uint32_t of(float v) {
        if constexpr (HALF) {
            const __half2 t = __float2half2_rn(v);
            return *reinterpret_cast<const uint32_t *>(&t);
        } else {
            const __nv_bfloat162 t = __float2bfloat162_rn(v);
            return *reinterpret_cast<const uint32_t *>(&t);
        }
    }
    static __device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) {
        if constexpr (HALF) {
            const __half2 t = __hadd2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
            return *reinterpret_cast<const uint32_t *>(&t);
        } else {
            const __nv_bfloat162 t = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
            return *reinterpret_cast<const uint32_t *>(&t);
        }
    }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c) {
        if constexpr (HALF) {
            const __half2 t = __hfma2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b), *reinterpret_cast<const __half2 *>(&c));
            return *reinterpret_cast<const uint32_t *>(&t);
        } else {
            const __nv_bfloat162 t = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b),
                                             *reinterpret_cast<const __nv_bfloat162 *>(&c));
            return *reinterpret_cast<const uint32_t *>(&t);
        }
    }
};

// How a type's pairs of B-bit codes are turned: positions 2^s a pair may stand at without a
// shift (s = 0, S, 2 S below LEVELS S), each with its own constant -(base / 2^s + z).
template <int B, bool HALF>
struct Turn {
    static constexpr int S = B;                                            // bits between neighbouring pairs
    static constexpr int LEVELS = B == 8 ? 1 : HALF ? (B == 4 ? 2 : 3) : (B == 2 ? 3 : B == 3 ? 2 : 1);
    using P = Pairs<HALF>;

    // -(base / 2^s + z): a float with z 2^s as its last bits
    static __device__ __forceinline__ void zero(uint32_t z, uint32_t (&k)[LEVELS]) {
        if constexpr (B == 8 && !HALF) {
            k[0] = P::of(-static_cast<float>(z));
        } else {
            constexpr uint32_t lead = P::kLead | 0x80008000u, step = HALF ? 0x04000400u : 0x00800080u;   // 1 of the exponent
#pragma unroll
            for (int i = 0; i < LEVELS; ++i) k[i] = z * (0x00010001u << (i * S)) + (lead - step * static_cast<uint32_t>(i * S));
        }
    }

    // pair number j (from bit 0) of a word
    static __device__ __forceinline__ uint32_t pair(uint32_t w, int j, const uint32_t (&k)[LEVELS]) {
        constexpr uint32_t mask = B == 8 ? 0x00ff00ffu : ((1u << B) - 1u) * 0x00010001u;
        if constexpr (B == 8) {
            if constexpr (HALF) {
                const uint32_t v = __byte_perm(w, 0x64646464u, j == 0 ? 0x4240 : 0x4341);   // 1024 + c
                return P::add(v, k[0]);
            } else {                                       // 16 upper + lower, both from 2^7
                const uint32_t lo = ((j ? w >> 8 : w) & 0x000f000fu) | P::kLead, hi = ((w >> (4 + 8 * j)) & 0x000f000fu) | P::kLead;
                const uint32_t l = P::add(lo, 0xC300C300u);                                  // less 128
                const uint32_t h = P::fma(hi, 0x41804180u, 0xC500C500u);                     // times 16, less 2048
                return P::add(P::add(h, l), k[0]);
            }
        } else {
            const int level = j % LEVELS, shift = (j - level) * S;
            const uint32_t v = ((w >> shift) & (mask << (level * S))) | P::kLead;
            return level == 0 ? P::add(v, k[0]) : P::fma(v, P::of(1.0f / static_cast<float>(1 << (level * S))), k[level]);
        }
    }

    // out[c][h][p]: c - z of the lane's pairs
    static __device__ __forceinline__ void unit(const uint32_t (&w)[B], const uint32_t (&k)[2][LEVELS], uint32_t (&out)[2][2][4]) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    if constexpr (B == 2) out[c][h][p] = pair(w[c], 4 * h + p, k[h]);
                    if constexpr (B == 4) out[c][h][p] = pair(w[2 * c + h], p, k[h]);
                    if constexpr (B == 8) out[c][h][p] = pair(w[4 * c + 2 * h + (p >> 1)], p & 1, k[h]);
                    if constexpr (B == 3) {
                        const int i = 8 * c + 4 * h + p;
                        if (i < 15) {
                            out[c][h][p] = pair(w[i / 5], i % 5, k[h]);
                        } else {
                            const uint32_t v = ((w[0] >> 15) & 0x00010001u) | ((w[1] >> 14) & 0x00020002u) | ((w[2] >> 13) & 0x00040004u) | P::kLead;
                            out[c][h][p] = P::add(v, k[h][0]);
                        }
                    }
                }
    }
};

// The word of zeros of a row tile's pair and a group; byte 2 i + h is row r + 8 h of row tile i of the pair.
__device__ __forceinline__ const uint32_t *zero_words(const LinearGeom &g, int tile, int r) {
    return g.zeros + static_cast<int64_t>(tile >> 1) * g.groups * 8 + r;
}
__device__ __forceinline__ uint32_t zero_of(uint32_t word, int byte) { return word >> (8 * byte) & 0xffu; }

__device__ __forceinline__ float to_f32(const void *p, int dtype, int64_t i) {
    if (dtype == QE_F32) return static_cast<const float *>(p)[i];
    if (dtype == QE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}

// Activations without branches, of __expf: by its stated bound off by (2 + 1.2 |a|) 2^-23 of the result for an exponent a, and the
// exponent's own rounding adds |a| 2^-24: 2^-20 of the result near 0, 2^-18 at a = -25, 2^-16 at -88, where binary32's exponentials end
// (a is y for SiLU, y^2 / 2 for GELU).  16 bits do not show it.  (With the library's erfc and quotients a tile's results took three times as long to leave as its products.)
// 1 / (1 + exp(-y)); far below 0 the 1 no longer counts and exp(-y) would leave binary32's range.
__device__ __forceinline__ float logistic(float y) { return y < -30.0f ? __expf(y) : __fdividef(1.0f, 1.0f + __expf(-y)); }

// Phi(y) = erfc(-y / sqrt 2) / 2, by the Chebyshev fit of erfc of Press et al., Numerical Recipes (relative error below
// 1.2e-7 everywhere): erfc(z) = t exp(-z^2 + P(t)), t = 1 / (1 + z / 2), z >= 0.
__device__ __forceinline__ float normal_cdf(float y) {
    const float z = 0.70710678118654752f * fabsf(y), t = __fdividef(1.0f, fmaf(0.5f, z, 1.0f));
    float p = 0.17087277f;
    p = fmaf(p, t, -0.82215223f);
    p = fmaf(p, t, 1.48851587f);
    p = fmaf(p, t, -1.13520398f);
    p = fmaf(p, t, 0.27886807f);
    p = fmaf(p, t, -0.18628806f);
    p = fmaf(p, t, 0.09678418f);
    p = fmaf(p, t, 0.37409196f);
    p = fmaf(p, t, 1.00002368f);
    p = fmaf(p, t, -1.26551223f);
    const float half = 0.5f * t * __expf(fmaf(-0.5f * y, y, p));
    return y < 0.0f ? half : 1.0f - half;
}

template <int ACT>
__device__ __forceinline__ float activated(float y) {
    if constexpr (ACT == QE_ACT_RELU) return y < 0.0f ? 0.0f : y;      // NaN stays
    if constexpr (ACT == QE_ACT_GELU) return y * normal_cdf(y);
    if constexpr (ACT == QE_ACT_GELU_TANH)                 // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return y * logistic(1.59576912160573072f * fmaf(0.044715f * y * y, y, y));
    if constexpr (ACT == QE_ACT_SILU) return y * logistic(y);
    return y;
}

// f of the call's activation as a constant.  (Chosen for each value instead, all of them were computed: a tile of 128 x 224
// results took 60000 cycles to leave, now 8000.)
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
        case QE_ACT_RELU: f(std::integral_constant<int, QE_ACT_RELU>{}); break;
        case QE_ACT_GELU: f(std::integral_constant<int, QE_ACT_GELU>{}); break;
        case QE_ACT_GELU_TANH: f(std::integral_constant<int, QE_ACT_GELU_TANH>{}); break;
        case QE_ACT_SILU: f(std::integral_constant<int, QE_ACT_SILU>{}); break;
        default: f(std::integral_constant<int, QE_ACT_NONE>{});
    }
}

// A finished sum (scaled) of output i for row m: bias, activation, residual, one rounding.
template <int ACT>
__device__ __forceinline__ void finish(const LinearArgs &a, float v, int64_t m, int64_t i, float bias) {
    v = activated<ACT>(v + bias);
    if (a.half) {
        if (a.residual) v += __half2float(static_cast<const __half *>(a.residual)[m * a.ldr + i]);
        static_cast<__half *>(a.y)[m * a.ldy + i] = __float2half_rn(v);
    } else {
        if (a.residual) v += __bfloat162float(static_cast<const __nv_bfloat16 *>(a.residual)[m * a.ldr + i]);
        static_cast<__nv_bfloat16 *>(a.y)[m * a.ldy + i] = __float2bfloat16_rn(v);
    }
}

// Raises a kernel's limit of dynamic shared memory on the current device, once a device; `raised`, a bit a device, is the
// kernel's own.  A refusal is not remembered.
inline cudaError_t raise_limit(const void *kernel, int bytes, std::atomic<uint64_t> &raised) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (raised.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Checks a layer and fills the geometry; QE_ERR_INVALID_ARG / QE_ERR_UNSUPPORTED otherwise.
qe_status linear_geom(const qe_layer *layer, LinearGeom *g);

// How the few-rows kernel is cut up: row tiles of a warp, CTAs that share a layer's columns.
struct RowsPlan {
    int tiles, ranks;
};
RowsPlan rows_plan(const LinearArgs &a);

// How the many-rows kernel is cut up: rows of x that its tiles have room for and have, CTAs that share a tile's columns.
struct TilesPlan {
    int room, rows, ranks;
};
TilesPlan tiles_plan(const LinearArgs &a);

int linear_sms();                         // of the current device

// few rows of x (and, slowly, any number of them), and many: x's address and pitch are then multiples of 16 bytes
cudaError_t launch_linear_rows_2(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_rows_3(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_rows_4(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_rows_8(const LinearArgs &a, cudaStream_t s);

cudaError_t launch_linear_tiles_2(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_tiles_3(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_tiles_4(const LinearArgs &a, cudaStream_t s);
cudaError_t launch_linear_tiles_8(const LinearArgs &a, cudaStream_t s);

}  // namespace qe
