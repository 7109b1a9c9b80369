// Norms of queries and keys, each head by itself, and their rotation by position.
//
//     y = x w / sqrt(mean(x^2) + eps);  (a, b) -> (a cos - b sin, b cos + a sin)
//
// A position's angles are phases in turns: position x (inv_freq / 2 pi mod 1), both whole
// numbers, the latter in units of 2^-64, is exact modulo one turn, where a binary32
// angle of 10^6 radians keeps a sixteenth of one.  The upper 32 bits give sin and cos of
// pi x, |x| < 1.
//
// Each channel is read and written once, which HBM bounds; in 16 bits what has to be issued comes close to it.  A lane has eight
// neighbouring channels (16 bytes of a 16-bit type) of a head in 8, 16 or 32 lanes, or four of either half where halves face each
// other; the mean meets in shuffles.  Two heads of a token go together (in 16 bits), binary32 arithmetic is on pairs, a block's
// tokens have their sines and cosines worked out once, for all heads.  Measured (us, TB/s read and written): 16384 tokens of 64
// heads of 128, bf16 105 (5.1), neighbouring pairs 107 (5.0); 8192 of 64, binary32 88 (6.1); 8192 of 240 heads of 64, fp16 90 (5.6);
// 8192 of 40 heads of 128 of which 36 channels turn 59 (2.8).  A head at a time and addresses by products: 122, 143, 86, 107, 107;
// blocks of 1, 2, 4, 8 and 16 tokens 137, 122, 113, 107, 107 (the first).
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "qe_cache.cuh"
#include "qe_internal.h"

namespace qe {
namespace {

constexpr int kMostPairs = 128, kBlockTokens = 8;

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
    int clear[2];             // whether tokens that are passed over get zeros
    int pairs, interleaved, facing;   // facing: pairs half a head apart face each other lane by lane
    uint64_t turns[kMostPairs];
};

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

// Pairs of binary32 numbers at once.
struct Two {
    uint64_t x;
};
__device__ __forceinline__ Two two(float lo, float hi) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.x) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void apart(Two v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v.x)); }
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.x) : "l"(a.x), "l"(b.x));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.x) : "l"(a.x), "l"(b.x), "l"(c.x));
    return r;
}

// Eight channels of a lane, rounded.
template <typename T>
__device__ __forceinline__ Eight<T> rounded_eight(const Two (&v)[4]) {
    Eight<T> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        apart(v[i], lo, hi);
        if constexpr (sizeof(T) == 4) {
            r.e[2 * i] = lo;
            r.e[2 * i + 1] = hi;
        } else if constexpr (std::is_same<T, __half>::value) {
            *reinterpret_cast<__half2 *>(r.e + 2 * i) = __floats2half2_rn(lo, hi);
        } else {
            *reinterpret_cast<__nv_bfloat162 *>(r.e + 2 * i) = __floats2bfloat162_rn(lo, hi);
        }
    }
    return r;
}

// A walk over a block's (token, head) pairs, `step` of them at a time: where the next one lies, without a product for each.
struct Walk {
    int64_t at, step_at, wrap_at;
    int t, h, step_t, step_h;
    __device__ __forceinline__ Walk(int first, int step, int heads, int64_t token, int64_t head) {
        t = first / heads;
        h = first - t * heads;
        step_t = step / heads;
        step_h = step - step_t * heads;
        at = t * token + h * head;
        step_at = step_t * token + step_h * head;
        wrap_at = token - heads * head;
    }
    __device__ __forceinline__ void next(int heads) {
        t += step_t;
        h += step_h;
        at += step_at;
        if (h >= heads) {
            ++t;
            h -= heads;
            at += wrap_at;
        }
    }
};

// Where a token's pair stands among its sines and cosines: pairs of neighbouring lanes side by side, `each` of them a lane.
__device__ __forceinline__ int turn_at(int p, int each, int stride) { return p % each * stride + p / each; }

// Heads of a token that a lane takes at once: what a pass costs besides its channels (where it lies, waiting, sines and cosines)
// is half of what is issued otherwise.
template <typename T>
constexpr int kHeads = sizeof(T) == 2 ? 2 : 1;

// grid: (groups of block_tokens tokens, shares of their heads, queries and keys); 256 threads.
// kSplit: the whole head turns, pairs half of it apart: a lane has four channels of either half, and its pairs to itself, as with
// kNeighbours, pairs of neighbouring channels (or none).  kAny: pairs in different lanes.
enum Form { kAny, kSplit, kNeighbours };

template <typename T, int LANES, Form FORM>
__global__ void __launch_bounds__(256, FORM == kAny ? 3 : 4) k_norm_rotate(const RotateArgs a) {
    constexpr bool SPLIT = FORM == kSplit;
    constexpr int AT_ONCE = 256 / LANES;                  // heads of a pass
    // sines and cosines: kAny [block_tokens][each][stride] of both, else [block_tokens][cos of all pairs, sin of all pairs], `room` each
    extern __shared__ __align__(16) float2 turned[];
    __shared__ __align__(16) float met[FORM == kAny ? 8 : 1][32 * 9];
    constexpr int kDeep = 3, kHead = 32 * 8 * sizeof(T), kSlot = kHeads<T> * kHead;
    __shared__ __align__(16) uint8_t ring[8][kDeep * kSlot];
    constexpr int each = FORM == kAny ? 8 : 4;            // pairs of a lane
    const int part = blockIdx.z, heads = a.heads[part], sets = (heads + kHeads<T> - 1) / kHeads<T>, stride = (a.pairs + each - 1) / each, room = stride * each;
    const int64_t tok0 = static_cast<int64_t>(blockIdx.x) * a.block_tokens;
    const int toks = a.tokens - tok0 < a.block_tokens ? static_cast<int>(a.tokens - tok0) : a.block_tokens;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = threadIdx.x % LANES, c0 = SPLIT ? 4 * sub : 8 * sub;
    const int upper_at = SPLIT ? a.pairs : 4;             // from a lane's first four channels to its second
    const bool mine = SPLIT ? c0 < a.pairs : c0 < a.dim;
    const int items = toks * sets, step = AT_ONCE * gridDim.y;
    // The warp's lanes go along together.  Heads come by asynchronous copies into a ring of
    // the warp's own, kDeep passes ahead and the first ones before the sines and cosines are worked out: in registers as many
    // bytes as that did not find room (145 us for 122 of the first size).
    const uint32_t ring0 = smem_u32(ring[warp]) + 8 * sizeof(T) * lane;
    const int first = blockIdx.y * AT_ONCE + warp * (32 / LANES) + lane / LANES;
    const T *x = static_cast<const T *>(a.x[part]) + tok0 * a.x_token[part] + 8 * sub;
    T *out = static_cast<T *>(a.out[part]) + tok0 * a.o_token[part] + c0;
    Walk from(first, step, sets, a.x_token[part], kHeads<T> * a.x_head[part]), to(first, step, sets, a.o_token[part], kHeads<T> * a.o_head[part]);
    uint32_t put = 0, get = 0;                            // offsets of slots
    int coming = 8 * sub < a.dim ? first : items;         // the item that comes next
    auto bring = [&]() {
        if (coming < items) {
#pragma unroll
            for (int j = 0; j < kHeads<T>; ++j) {
                if (j > 0 && kHeads<T> * from.h + j >= heads) break;
                const T *p = x + from.at + j * a.x_head[part];
                if ((a.vec & 1) != 0) {
#pragma unroll
                    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring0 + put + j * kHead + 16 * i),
                                     "l"(reinterpret_cast<uint64_t>(p) + 16 * i)
                                     : "memory");
                } else {
                    T *place = reinterpret_cast<T *>(ring[warp] + put + j * kHead) + 8 * lane;
#pragma unroll
                    for (int i = 0; i < 8; ++i) place[i] = p[i];
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        coming += step;
        from.next(sets);
        put = put == (kDeep - 1) * kSlot ? 0 : put + kSlot;
    };
#pragma unroll
    for (int k = 0; k < kDeep - 1; ++k) bring();
    for (int i = threadIdx.x; i < toks * room; i += 256) {
        const int t = i / room, p = i - t * room;
        float s = 0.0f, c = 1.0f;                         // (of a pair that is not there: no turn)
        if (p < a.pairs) {
            const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(a.positions[tok0 + t])) * a.turns[p];
            sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 4.656612873077392578125e-10f, &s, &c);   // 2^-31
        }
        if constexpr (FORM == kAny) {
            turned[t * room + turn_at(p, each, stride)] = make_float2(c, s);
        } else {
            float *cs = reinterpret_cast<float *>(turned + t * room) + p;
            cs[0] = c;
            cs[room] = s;
        }
    }
    unsigned live = 0u;                                   // tokens whose position is not negative
    for (int t = 0; t < toks; ++t) live |= static_cast<unsigned>(!a.positions || a.positions[tok0 + t] >= 0) << t;
    if (a.clear[part] && live != (1u << toks) - 1u) {     // (beside the loop: in it, 109 us for the first size's 105)
        Walk at = to;
        for (int it = first; it < items; it += step, at.next(sets))
            if (mine && !(live >> at.t & 1u))
                for (int j = 0; j < kHeads<T> && kHeads<T> * at.h + j < heads; ++j)
                    store_eight<T, SPLIT>(out + at.at + j * a.o_head[part], (a.vec & 2) != 0, upper_at, Eight<T>{});
    }
    Two w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = c0 + (i >> 1) * upper_at + 2 * (i & 1);
        const bool on = a.weight[part] && mine;
        w[i] = two(on ? weight_at(a.weight[part], a.weight_dtype, c) : 1.0f, on ? weight_at(a.weight[part], a.weight_dtype, c + 1) : 1.0f);
    }
    __syncthreads();
    const int half = a.pairs, most = 2 * a.pairs;
    for (int it = first; it - lane / LANES < items; it += step, to.next(sets), get = get == (kDeep - 1) * kSlot ? 0 : get + kSlot) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 2) : "memory");
        __syncwarp();                                     // every lane's copies of the pass are there, the pass before has been read
        bring();
        const int t = it < items ? to.t : 0;              // (of an item that is not there nothing is stored)
        ulonglong2 cc = make_ulonglong2(0, 0), ss = cc;
        const int c_at = SPLIT ? (mine ? c0 : 0) : c0 / 2;   // the lane's first pair
        const bool turns = SPLIT || (FORM == kNeighbours && c_at < a.pairs);
        if (turns) {
            const float *cs = reinterpret_cast<const float *>(turned + t * room) + c_at;
            cc = *reinterpret_cast<const ulonglong2 *>(cs);
            ss = *reinterpret_cast<const ulonglong2 *>(cs + room);
        }
#pragma unroll
        for (int j = 0; j < kHeads<T>; ++j) {             // (a second head that is not there is not stored)
            const T *head = reinterpret_cast<const T *>(ring[warp] + get + j * kHead) + 8 * (lane - sub) + c0;
            const Eight<T> raw = load_eight<T, SPLIT>(mine ? head : head - c0, true, mine ? upper_at : 4);
            Two v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = two(static_cast<float>(raw.e[2 * i]), static_cast<float>(raw.e[2 * i + 1]));
            if (a.weight[part]) {
                Two both = mul2(v[0], v[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) both = fma2(v[i], v[i], both);
                float sum, odd;
                apart(both, sum, odd);
                sum = mine ? sum + odd : 0.0f;
#pragma unroll
                for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float by = rsqrtf(fmaf(sum, a.per_dim, a.eps));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], mul2(two(by, by), w[i]));
            }
            if constexpr (SPLIT) {
                const Two less = two(-1.0f, -1.0f), c2[2] = {{cc.x}, {cc.y}}, s2[2] = {{ss.x}, {ss.y}};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const Two p = v[i], q = v[i + 2];
                    v[i] = fma2(mul2(q, s2[i]), less, mul2(p, c2[i]));
                    v[i + 2] = fma2(p, s2[i], mul2(q, c2[i]));
                }
            } else if constexpr (FORM == kNeighbours) {
                float c[4], s[4];
                apart(Two{cc.x}, c[0], c[1]);
                apart(Two{cc.y}, c[2], c[3]);
                apart(Two{ss.x}, s[0], s[1]);
                apart(Two{ss.y}, s[2], s[3]);
                if (turns)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float p, q;
                        apart(v[i], p, q);
                        v[i] = two(p * c[i] - q * s[i], q * c[i] + p * s[i]);
                    }
            } else {
                const float2 *cs = turned + t * room;
                float u[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) apart(v[i], u[2 * i], u[2 * i + 1]);
                if (a.facing) {
                    const bool turns = c0 < most, upper = c0 >= half;   // (of the lane's channels)
                    const int face = turns ? (upper ? lane - half / 8 : lane + half / 8) : lane;
                    const float2 *mine_cs = cs + (turns ? (upper ? c0 - half : c0) >> 3 : 0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float q = __shfl_sync(0xffffffffu, u[i], face);
                        const float2 r = mine_cs[i * stride];
                        if (turns) u[i] = fmaf(upper ? q : -q, r.y, u[i] * r.x);
                    }
                } else {
                    float *place = met[warp] + (lane - sub) * 9;  // the head's channel c at c + c / 8
#pragma unroll
                    for (int i = 0; i < 8; ++i) place[sub * 9 + i] = u[i];
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = c0 + i;
                        if (c < most) {
                            const bool upper = c >= half;
                            const int other = upper ? c - half : c + half;
                            const float q = place[other + other / 8];
                            const float2 r = cs[turn_at(upper ? c - half : c, each, stride)];
                            u[i] = fmaf(upper ? q : -q, r.y, u[i] * r.x);
                        }
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = two(u[2 * i], u[2 * i + 1]);
            }
            if (it < items && mine && (live >> t & 1u) && (j == 0 || kHeads<T> * to.h + j < heads))
                store_eight<T, SPLIT>(out + to.at + j * a.o_head[part], (a.vec & 2) != 0, upper_at, rounded_eight<T>(v));
        }
    }
}

template <typename T, int LANES, Form FORM>
cudaError_t launch_lanes(const RotateArgs &a, cudaStream_t s) {
    const int most = ((a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1]) + kHeads<T> - 1) / kHeads<T>;
    const int64_t groups = ceil_div(a.tokens, a.block_tokens);
    // few tokens: their heads are shared out over blocks, a pass each, up to four blocks an SM
    const int passes = static_cast<int>(ceil_div(static_cast<int64_t>(a.block_tokens) * most, 256 / LANES));
    int64_t shares = 608 / groups;                        // (four blocks an SM)
    shares = shares < 1 ? 1 : shares > passes ? passes : shares;
    const int first = a.heads[0] > 0 ? 0 : 1;             // (a call without queries has one part as well)
    RotateArgs b = a;
    if (first == 1) {
        b.x[0] = a.x[1]; b.out[0] = a.out[1]; b.weight[0] = a.weight[1]; b.heads[0] = a.heads[1];
        b.clear[0] = a.clear[1];
        b.x_token[0] = a.x_token[1]; b.x_head[0] = a.x_head[1]; b.o_token[0] = a.o_token[1]; b.o_head[0] = a.o_head[1];
        b.heads[1] = 0;
    }
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>(shares), b.heads[1] > 0 ? 2 : 1);
    const int room = static_cast<int>(round_up(a.pairs, FORM == kAny ? 8 : 4));
    k_norm_rotate<T, LANES, FORM><<<grid, 256, static_cast<size_t>(a.block_tokens) * room * sizeof(float2), s>>>(b);
    return cudaGetLastError();
}

template <typename T, Form FORM>
cudaError_t launch_form(const RotateArgs &a, cudaStream_t s) {
    if (a.dim <= 64) return launch_lanes<T, 8, FORM>(a, s);
    return a.dim <= 128 ? launch_lanes<T, 16, FORM>(a, s) : launch_lanes<T, 32, FORM>(a, s);
}

template <typename T>
cudaError_t launch_type(const RotateArgs &a, cudaStream_t s) {
    if (a.interleaved || a.pairs == 0) return launch_form<T, kNeighbours>(a, s);
    return 2 * a.pairs == a.dim && a.pairs % 4 == 0 ? launch_form<T, kSplit>(a, s) : launch_form<T, kAny>(a, s);
}

bool aligned16(const void *p, int64_t a, int64_t b, size_t size) {
    const int64_t n = static_cast<int64_t>(16 / size);
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && a % n == 0 && b % n == 0;
}

// t modulo 1, times 2^64, to the nearest.  A magnitude's fraction is exact, which 1 less a small one's would not be.
uint64_t fraction(double t) {
    const double m = fabs(t), part = ldexp(m - floor(m), 32), upper = floor(part);
    const uint64_t turns = (static_cast<uint64_t>(upper) << 32) + static_cast<uint64_t>(rint(ldexp(part - upper, 32)));
    return t < 0.0 ? 0 - turns : turns;
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
        (h->weight_dtype != QE_F32 && h->weight_dtype != QE_BF16 && h->weight_dtype != QE_F16) || !(h->eps >= 0.0f) || isinf(h->eps) || (h->clear & ~3) != 0)
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
    a.clear[0] = h->clear & 1; a.clear[1] = h->clear >> 1 & 1;
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
    // Up to eight tokens a block, while that still gives every SM four blocks.  Measured (us, one a block / so many; 64 heads of 128,
    // bf16): 1300 tokens 20 / 18, 2000 27 / 20, 2500 33 / 25, 3500 43 / 31, 4800 55 / 39; 16384, 4 / 8 / 16: 113 / 107 / 107.
    a.block_tokens = static_cast<int>(h->tokens >= 608 * kBlockTokens ? kBlockTokens : h->tokens >= 1216 ? h->tokens / 608 : 1);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = h->dtype == QE_F32 ? launch_type<float>(a, s) : h->dtype == QE_BF16 ? launch_type<__nv_bfloat16>(a, s) : launch_type<__half>(a, s);
    return e == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

}  // extern "C"
