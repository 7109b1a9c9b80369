// Norms of queries and keys, each head by itself, and their rotation by position.
//
//     y = x w / sqrt(mean(x^2) + eps);  (a, b) -> (a cos - b sin, b cos + a sin)
//
// A position's angles are phases in turns: position x (inv_freq / 2 pi mod 1), both whole
// numbers, the latter in units of 2^-64, is exact modulo one turn, where a binary32
// angle of 10^6 radians keeps a sixteenth of one.  The upper 32 bits give sin and cos of
// pi x, |x| < 1.
//
// Bound by HBM: each channel is read and written once.  A lane has eight neighbouring
// channels (16 bytes of a 16-bit type) of a head in 8, 16 or 32 lanes, the mean meets in
// shuffles and so do pairs that lie half a head apart (through shared memory where a lane's
// eight do not face another lane's).  A block's tokens have their sines and cosines worked out once,
// for all heads.
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "qe_cache.cuh"
#include "qe_internal.h"

namespace qe {
namespace {

constexpr int kMostPairs = 128, kBlockTokens = 4;

struct RotateArgs {
    const void *x[2];         // queries, keys
    void *out[2];
    const void *weight[2];
    int64_t x_token[2], x_head[2], o_token[2], o_head[2];
    int heads[2];
    int vec;                  // 16-byte accesses are aligned (bits: loads, stores, weights)
    int64_t tokens;
    int dim, block_tokens, weight_dtype;
    float eps, per_dim;
    const int32_t *positions;
    int pairs, interleaved, facing;   // facing: pairs half a head apart face each other lane by lane
    uint64_t turns[kMostPairs];
};

template <typename T>
__device__ __forceinline__ T rounded_to(float v);
template <>
__device__ __forceinline__ float rounded_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half rounded_to<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 rounded_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float weight_at(const void *w, int dtype, int i) {
    if (dtype == QE_F32) return static_cast<const float *>(w)[i];
    if (dtype == QE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[i]);
    return __half2float(static_cast<const __half *>(w)[i]);
}

// Eight channels as they lie in memory.
template <typename T>
struct alignas(16) Eight {
    T e[8];
};

// A lane's four channels from p on, and the four `upper` further (at once where they are neighbours).
template <typename T, bool SPLIT>
__device__ __forceinline__ Eight<T> load_eight(const T *p, bool vec, int upper) {
    using Four = typename std::conditional<sizeof(T) == 2, uint2, uint4>::type;
    Eight<T> r;
    if (vec && SPLIT) {
        reinterpret_cast<Four *>(r.e)[0] = *reinterpret_cast<const Four *>(p);
        reinterpret_cast<Four *>(r.e)[1] = *reinterpret_cast<const Four *>(p + upper);
    } else if (vec) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4 *>(r.e)[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.e[i] = p[(i & 3) + (i >> 2) * upper];
    }
    return r;
}

template <typename T, bool SPLIT>
__device__ __forceinline__ void store_eight(T *p, bool vec, int upper, const Eight<T> &r) {
    using Four = typename std::conditional<sizeof(T) == 2, uint2, uint4>::type;
    if (vec && SPLIT) {
        *reinterpret_cast<Four *>(p) = reinterpret_cast<const Four *>(r.e)[0];
        *reinterpret_cast<Four *>(p + upper) = reinterpret_cast<const Four *>(r.e)[1];
    } else if (vec) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(r.e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[(i & 3) + (i >> 2) * upper] = r.e[i];
    }
}

// Where a token's pair stands among its sines and cosines: pairs of neighbouring lanes side by side, `each` of them a lane.
__device__ __forceinline__ int turn_at(int p, int each, int stride) { return p % each * stride + p / each; }

// grid: (groups of block_tokens tokens, shares of their heads, queries and keys); 256 threads.
// SPLIT: the whole head turns, pairs half of it apart: a lane has four channels of either half, and its pairs to itself.
template <typename T, int LANES, bool SPLIT>
__global__ void __launch_bounds__(256, SPLIT ? 5 : 4) k_norm_rotate(const RotateArgs a) {
    constexpr int AT_ONCE = 256 / LANES;                  // heads of a pass
    extern __shared__ __align__(16) float2 turned[];      // [block_tokens][each][stride]: cos, sin
    __shared__ __align__(16) float met[SPLIT ? 1 : 8][32 * 9];
    constexpr int kDeep = sizeof(T) == 2 ? 4 : 3, kSlot = 32 * 8 * sizeof(T);
    __shared__ __align__(16) uint8_t ring[8][kDeep * kSlot];
    __shared__ int live[kBlockTokens];                    // not a negative position's
    const int each = SPLIT || a.interleaved ? 4 : 8;      // pairs of a lane
    const int part = blockIdx.z, heads = a.heads[part], stride = (a.pairs + each - 1) / each;
    const int64_t tok0 = static_cast<int64_t>(blockIdx.x) * a.block_tokens;
    const int toks = a.tokens - tok0 < a.block_tokens ? static_cast<int>(a.tokens - tok0) : a.block_tokens;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = threadIdx.x % LANES, c0 = SPLIT ? 4 * sub : 8 * sub;
    const int upper_at = SPLIT ? a.pairs : 4;             // from a lane's first four channels to its second
    const bool mine = SPLIT ? c0 < a.pairs : c0 < a.dim;
    const T *x = static_cast<const T *>(a.x[part]) + tok0 * a.x_token[part];
    T *out = static_cast<T *>(a.out[part]) + tok0 * a.o_token[part];
    const int items = toks * heads, step = AT_ONCE * gridDim.y;
    // The warp's lanes go along together; `item` is the warp's first head's.  Heads come by asynchronous copies into a ring of
    // the warp's own, kDeep passes ahead and the first ones before the sines and cosines are worked out: in registers as many
    // bytes as that did not find room (16384 tokens of 64 heads of 128, bf16: 145 us).
    const uint32_t slot0 = smem_u32(ring[warp]), mine_at = 8 * sizeof(T) * lane;
    const int copy_c = 8 * sub;
    const int first = blockIdx.y * AT_ONCE + warp * (32 / LANES);
    auto bring = [&](int pass) {
        const int it = first + pass * step + lane / LANES;
        const uint32_t to = slot0 + (pass % kDeep) * kSlot + mine_at;
        if (it < items && copy_c < a.dim) {
            const int t = (it >= heads) + (it >= 2 * heads) + (it >= 3 * heads);          // of up to kBlockTokens
            const T *from = x + t * a.x_token[part] + (it - t * heads) * a.x_head[part] + copy_c;
            if ((a.vec & 1) != 0) {
#pragma unroll
                for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16 * i), "l"(reinterpret_cast<uint64_t>(from) + 16 * i) : "memory");
            } else {
                T *p = reinterpret_cast<T *>(ring[warp] + (pass % kDeep) * kSlot + mine_at);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = from[i];
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kDeep - 1; ++k) bring(k);
    for (int i = threadIdx.x; i < toks * a.pairs; i += 256) {
        const int t = i / a.pairs, p = i - t * a.pairs;
        const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(a.positions[tok0 + t])) * a.turns[p];
        float s, c;
        sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 4.656612873077392578125e-10f, &s, &c);   // 2^-31
        turned[t * each * stride + turn_at(p, each, stride)] = make_float2(c, s);
    }
    if (threadIdx.x < toks) live[threadIdx.x] = !a.positions || a.positions[tok0 + threadIdx.x] >= 0;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = a.weight[part] && mine ? weight_at(a.weight[part], a.weight_dtype, c0 + (i & 3) + (i >> 2) * upper_at) : 1.0f;
    __syncthreads();
    const int half = a.pairs, most = 2 * a.pairs;
    for (int pass = 0; first + pass * step < items; ++pass) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 2) : "memory");
        __syncwarp();                                     // every lane's copies of the pass are there, the pass before has been read
        bring(pass + kDeep - 1);
        const int it = first + pass * step + lane / LANES;
        const bool on = it < items && mine;
        const int t = it < items ? (it >= heads) + (it >= 2 * heads) + (it >= 3 * heads) : 0, h = it < items ? it - t * heads : 0;
        const T *head = reinterpret_cast<const T *>(ring[warp] + (pass % kDeep) * kSlot) + 8 * (lane - sub) + c0;
        const Eight<T> raw = load_eight<T, SPLIT>(mine ? head : head - c0, true, mine ? upper_at : 4);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = on ? static_cast<float>(raw.e[i]) : 0.0f;
        {
            if (a.weight[part]) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
#pragma unroll
                for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float by = rsqrtf(fmaf(sum, a.per_dim, a.eps));
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= by * w[i];
            }
            const float2 *cs = turned + t * each * stride;
            if constexpr (SPLIT) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 r = cs[i * stride + (mine ? sub : 0)];
                    const float p = v[i], q = v[i + 4];
                    v[i] = p * r.x - q * r.y;
                    v[i + 4] = q * r.x + p * r.y;
                }
            } else if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; i += 2)
                    if (c0 + i < most) {
                        const float2 r = cs[(i >> 1) * stride + sub];
                        const float p = v[i], q = v[i + 1];
                        v[i] = p * r.x - q * r.y;
                        v[i + 1] = q * r.x + p * r.y;
                    }
            } else if (a.facing) {
                const bool turns = c0 < most, upper = c0 >= half;
                const int face = turns ? (upper ? lane - half / 8 : lane + half / 8) : lane;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float q = __shfl_sync(0xffffffffu, v[i], face);
                    if (turns) {
                        const float2 r = cs[i * stride + ((upper ? c0 - half : c0) >> 3)];
                        v[i] = upper ? v[i] * r.x + q * r.y : v[i] * r.x - q * r.y;
                    }
                }
            } else if (most > 0) {
                float *place = met[warp] + (lane - sub) * 9;  // the head's channel c at c + c / 8
#pragma unroll
                for (int i = 0; i < 8; ++i) place[sub * 9 + i] = v[i];
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = c0 + i;
                    if (c < most) {
                        const bool upper = c >= half;
                        const int other = upper ? c - half : c + half;
                        const float q = place[other + other / 8];
                        const float2 r = cs[turn_at(upper ? c - half : c, each, stride)];
                        v[i] = upper ? v[i] * r.x + q * r.y : v[i] * r.x - q * r.y;
                    }
                }
                __syncwarp();
            }
            if (on && live[t]) {
                Eight<T> r;
#pragma unroll
                for (int i = 0; i < 8; ++i) r.e[i] = rounded_to<T>(v[i]);
                store_eight<T, SPLIT>(out + t * a.o_token[part] + h * a.o_head[part] + c0, (a.vec & 2) != 0, upper_at, r);
            }
        }
    }
}

template <typename T, int LANES, bool SPLIT>
cudaError_t launch_lanes(const RotateArgs &a, cudaStream_t s) {
    const int most = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1];
    const int64_t groups = ceil_div(a.tokens, a.block_tokens);
    // few tokens: their heads are shared out over blocks, a pass each, up to four blocks an SM
    const int passes = static_cast<int>(ceil_div(static_cast<int64_t>(a.block_tokens) * most, 256 / LANES));
    int64_t shares = 608 / groups;                        // (four blocks an SM)
    shares = shares < 1 ? 1 : shares > passes ? passes : shares;
    const int first = a.heads[0] > 0 ? 0 : 1;             // (a call without queries has one part as well)
    RotateArgs b = a;
    if (first == 1) {
        b.x[0] = a.x[1]; b.out[0] = a.out[1]; b.weight[0] = a.weight[1]; b.heads[0] = a.heads[1];
        b.x_token[0] = a.x_token[1]; b.x_head[0] = a.x_head[1]; b.o_token[0] = a.o_token[1]; b.o_head[0] = a.o_head[1];
        b.heads[1] = 0;
    }
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>(shares), b.heads[1] > 0 ? 2 : 1);
    const int each = SPLIT || a.interleaved ? 4 : 8, room = static_cast<int>(round_up(a.pairs, each));
    k_norm_rotate<T, LANES, SPLIT><<<grid, 256, static_cast<size_t>(a.block_tokens) * room * sizeof(float2), s>>>(b);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const RotateArgs &a, cudaStream_t s) {
    if (2 * a.pairs == a.dim && !a.interleaved && a.pairs % 4 == 0) {
        if (a.dim <= 64) return launch_lanes<T, 8, true>(a, s);
        return a.dim <= 128 ? launch_lanes<T, 16, true>(a, s) : launch_lanes<T, 32, true>(a, s);
    }
    if (a.dim <= 64) return launch_lanes<T, 8, false>(a, s);
    return a.dim <= 128 ? launch_lanes<T, 16, false>(a, s) : launch_lanes<T, 32, false>(a, s);
}

bool aligned16(const void *p, int64_t a, int64_t b, size_t size) {
    const int64_t n = static_cast<int64_t>(16 / size);
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && a % n == 0 && b % n == 0;
}

// t modulo 1, times 2^64.
uint64_t fraction(double t) {
    t = ldexp(t - floor(t), 32);                          // 0 .. 2^32 (the end: by rounding, no turn at all)
    const double upper = floor(t);
    return (static_cast<uint64_t>(upper) << 32) + static_cast<uint64_t>(ldexp(t - upper, 32));
}

}  // namespace
}  // namespace qe

using namespace qe;

extern "C" {

qe_status qe_rope_init(const double *inv_freq, int pairs, int interleaved, qe_rope *rope) {
    if (!inv_freq || !rope || pairs < 1 || pairs > kMostPairs) return QE_ERR_INVALID_ARG;
    for (int i = 0; i < pairs; ++i)
        if (!isfinite(inv_freq[i])) return QE_ERR_INVALID_ARG;
    rope->pairs = pairs;
    rope->interleaved = interleaved != 0;
    for (int i = 0; i < kMostPairs; ++i) {
        rope->turns[i] = 0;
        if (i >= pairs) continue;
        // the quotient by 2 pi in two doubles
        const double two_pi = 6.283185307179586476925, rest = 2.4492935982947064e-16, f = inv_freq[i];   // two_pi + rest = 2 pi
        const double upper = f / two_pi, lower = (fma(-upper, two_pi, f) - upper * rest) / two_pi;
        rope->turns[i] = fraction(upper) + fraction(lower);
    }
    return QE_OK;
}

qe_status qe_norm_rotate(const qe_heads *h, qe_stream_t stream) {
    if (!h || h->tokens < 0 || h->tokens > 0x7fffffff || h->q_heads < 0 || h->k_heads < 0 || h->q_heads > 65535 || h->k_heads > 65535)
        return QE_ERR_INVALID_ARG;
    if (h->head_dim < 8) return QE_ERR_INVALID_ARG;
    if (h->head_dim > 256 || h->head_dim % 8 != 0) return QE_ERR_UNSUPPORTED;
    if ((h->dtype != QE_F32 && h->dtype != QE_BF16 && h->dtype != QE_F16) ||
        (h->weight_dtype != QE_F32 && h->weight_dtype != QE_BF16 && h->weight_dtype != QE_F16) || !(h->eps >= 0.0f) || isinf(h->eps))
        return QE_ERR_INVALID_ARG;
    if (h->rope && (h->rope->pairs < 1 || h->rope->pairs > kMostPairs || 2 * h->rope->pairs > h->head_dim)) return QE_ERR_INVALID_ARG;
    if (h->tokens == 0 || (h->q_heads == 0 && h->k_heads == 0)) return QE_OK;
    const size_t size = h->dtype == QE_F32 ? 4 : 2, wsize = h->weight_dtype == QE_F32 ? 4 : 2;
    RotateArgs a{};
    a.x[0] = h->Q; a.x[1] = h->K; a.out[0] = h->q_out; a.out[1] = h->k_out;
    a.weight[0] = h->q_weight; a.weight[1] = h->k_weight;
    a.x_token[0] = h->q_token; a.x_token[1] = h->k_token; a.x_head[0] = h->q_head; a.x_head[1] = h->k_head;
    a.o_token[0] = h->qo_token; a.o_token[1] = h->ko_token; a.o_head[0] = h->qo_head; a.o_head[1] = h->ko_head;
    a.heads[0] = h->q_heads; a.heads[1] = h->k_heads;
    a.vec = 3;
    for (int i = 0; i < 2; ++i) {
        if (a.heads[i] == 0) continue;
        if (!a.x[i] || !a.out[i] || reinterpret_cast<uintptr_t>(a.x[i]) % size != 0 || reinterpret_cast<uintptr_t>(a.out[i]) % size != 0 ||
            reinterpret_cast<uintptr_t>(a.weight[i]) % wsize != 0)
            return QE_ERR_INVALID_ARG;
        if (!aligned16(a.x[i], a.x_token[i], a.x_head[i], size)) a.vec &= ~1;
        if (!aligned16(a.out[i], a.o_token[i], a.o_head[i], size)) a.vec &= ~2;
    }
    if ((h->rope && !h->positions) || (reinterpret_cast<uintptr_t>(h->positions) & 3u) != 0) return QE_ERR_INVALID_ARG;
    a.tokens = h->tokens;
    a.dim = h->head_dim;
    a.weight_dtype = h->weight_dtype;
    a.eps = h->eps;
    a.per_dim = 1.0f / static_cast<float>(h->head_dim);
    a.positions = h->positions;
    if (h->rope) {
        a.pairs = h->rope->pairs;
        a.interleaved = h->rope->interleaved != 0;
        a.facing = a.pairs % 8 == 0;
        for (int i = 0; i < a.pairs; ++i) a.turns[i] = h->rope->turns[i];
    }
    a.block_tokens = h->tokens >= 2432 ? kBlockTokens : 1;         // four tokens a block where that still gives every SM four blocks
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = h->dtype == QE_F32 ? launch_type<float>(a, s) : h->dtype == QE_BF16 ? launch_type<__nv_bfloat16>(a, s) : launch_type<__half>(a, s);
    return e == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

}  // extern "C"
