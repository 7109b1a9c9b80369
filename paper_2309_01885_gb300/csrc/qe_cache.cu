// Writing the 4-bit key/value cache and reading it back (layout: qe_cache.cuh).
//
// Both kernels give eight channels of a token's head to a lane: 16 bytes of a 16-bit
// type, one word of key codes, two halves of value codes.  A block takes 16 or 32
// tokens of the call's list for one head, so that the value words that neighbouring
// tokens share meet in L1, and two tokens whose slots make a pair exchange halves and
// move whole words.  A group's minimum and maximum meet in shuffles.  Bound by HBM: 2 +
// 0.5 + 4 / G bytes for each 16-bit channel.  Measured: 32768 tokens, 8 heads of 128, read
// back in 37 us (4.6 TB/s, kernel and call); 16384 tokens, 32 heads of 128, written in 119
// us (2.9 TB/s: minima, maxima, one exact rounding and one code a channel fill 75% of the
// issue slots) and read in 64 (5.4 TB/s).  A few tokens take 2 to 4 us on the GPU.
#include <cuda_fp16.h>

#include <type_traits>

#include "qe_cache.cuh"
#include "qe_internal.h"

namespace qe {

qe_status cache_geom(const qe_cache *c, CacheGeom *g) {
    if (!c || !c->data || (reinterpret_cast<uintptr_t>(c->data) & 255u) != 0) return QE_ERR_INVALID_ARG;
    size_t need = 0;
    const qe_status st = qe_cache_size(c->pages, c->page_size, c->kv_heads, c->head_dim, c->group_size, &need);
    if (st != QE_OK) return st;
    if (c->bytes < need) return QE_ERR_INVALID_ARG;
    g->data = static_cast<uint8_t *>(c->data);
    g->pages = c->pages;
    g->page_shift = 31 - __builtin_clz(static_cast<unsigned>(c->page_size));
    g->kv_heads = c->kv_heads;
    g->dim = c->head_dim;
    g->D = cache_padded(c->head_dim);
    g->group_shift = 31 - __builtin_clz(static_cast<unsigned>(c->group_size));
    g->groups = g->D / c->group_size;
    g->block_bytes = static_cast<uint32_t>(g->D + 8 * g->groups) * static_cast<uint32_t>(c->page_size);
    g->page_bytes = g->block_bytes * static_cast<uint32_t>(c->kv_heads);
    g->v_off = static_cast<uint32_t>(g->D / 2) << g->page_shift;
    g->kg_off = static_cast<uint32_t>(g->D) << g->page_shift;
    g->vg_off = static_cast<uint32_t>(g->D + 4 * g->groups) << g->page_shift;
    return QE_OK;
}

namespace {

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Eight neighbouring channels and their extremes with 0; `vec`: 16-byte accesses are aligned.
template <typename T>
__device__ __forceinline__ void load8(const T *p, bool vec, float (&v)[8], float &lo, float &hi) {
    union { uint4 u[sizeof(T) / 2]; T e[8]; } t;
    if (vec) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) t.u[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) t.e[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(t.e[i]);
    if constexpr (sizeof(T) == 2) {                       // two at a time
        using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const T2 *e = reinterpret_cast<const T2 *>(t.e);
        const T2 a = __hmin2(__hmin2(e[0], e[1]), __hmin2(e[2], e[3])), b = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
        lo = fminf(0.0f, fminf(static_cast<float>(a.x), static_cast<float>(a.y)));
        hi = fmaxf(0.0f, fmaxf(static_cast<float>(b.x), static_cast<float>(b.y)));
    } else {
        lo = hi = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo = fminf(lo, v[i]);
            hi = fmaxf(hi, v[i]);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, bool vec, const T (&v)[8]) {
    union { uint4 u[sizeof(T) / 2]; T e[8]; } t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.e[i] = v[i];
    if (vec) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = t.u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = t.e[i];
    }
}

// round(x / s), ties to even, left in the low bits of a sum with 1.5 2^23 (whose addition rounds so).
//
// x / s is taken as q = x (1 / s), at most 3 units in the last place off, which only matters next to a midpoint h
// between two integers.  With 16-bit x, x and s h are both multiples of 2^-13 of their size (11 bits of x; 8 of s
// times 5 of 2 h): x / s is h itself or at least 2^-14 away, and rounding q to multiples of 2^-16 first (as the sum
// with 192 does) puts it on h in the one case and leaves it on its side in the other.  Binary32 x are divided
// where q lies next to a midpoint.
constexpr float kRound = 12582912.0f;
template <typename T, int N>
__device__ __forceinline__ void rounded(const float (&x)[N], float s, float (&t)[N]) {
    const float inv = __frcp_rn(s);                       // s >= 2^-126: at most 2^126
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = __fadd_rn(__fmaf_rn(x[i], inv, 192.0f), kRound - 192.0f);
    } else {
        float off = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float q = x[i] * inv;
            t[i] = __fadd_rn(q, kRound);
            off = fmaxf(off, fabsf(q - __fsub_rn(t[i], kRound)));
        }
        if (off > 0.49999f)
#pragma unroll
            for (int i = 0; i < N; ++i) t[i] = __fadd_rn(__fdiv_rn(x[i], s), kRound);
    }
}

// clamp(round(x / s) + z, 0, 15) for eight channels, code i at bit shift(i).  No code falls below 0: z is
// round(-lo / s), and rounding keeps order and sign.
template <typename T, typename Shift>
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float s, float z, Shift shift) {
    float t[8];
    rounded<T>(x, s, t);
    uint32_t w = 0u, base = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w += __float_as_uint(fminf(__fadd_rn(t[i], z), kRound + 15.0f)) << shift(i);
        base += 0x4B400000u << shift(i);
    }
    return w - base;
}

// The grid of a group whose channels lie in `lanes` neighbouring lanes (eight each), from the lane's own extremes.
template <typename T>
__device__ __forceinline__ void group_grid(float lo, float hi, int lanes, float &s, float &z) {
    for (int o = 1; o < lanes; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const float r = __fdiv_rn(__fsub_rn(hi, lo), 15.0f);
    s = fmaxf(__bfloat162float(__float2bfloat16_rn(r)), 1.17549435e-38f);
    const float x[1] = {-lo};
    float t[1];
    rounded<T>(x, s, t);
    z = __fsub_rn(t[0], kRound);
}

// Eight channels' s (c - z), rounded once to T, from pairs of codes at bits 0 and 16 of p[0 .. 3]; c - z is exact.
template <typename T>
__device__ __forceinline__ void values8(const uint32_t (&p)[4], uint32_t grid, T (&out)[8]) {
    const float s = __uint_as_float(grid & 0xFFFF0000u), z = __uint_as_float(grid << 16);
    if constexpr (sizeof(T) == 2 && !std::is_same<T, __half>::value) {
        // the scale is a bf16 number: one product in bf16 rounds as the definition does
        const __nv_bfloat162 s2 = __float2bfloat162_rn(s), z2 = __float2bfloat162_rn(z + 128.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = p[i] | 0x43004300u;        // 128 + c
            const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&w), z2), s2);
            out[2 * i] = v.x;
            out[2 * i + 1] = v.y;
        }
    } else {
        const __half2 z2 = __float2half2_rn(z + 1024.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = p[i] | 0x64006400u;        // 1024 + c
            const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&w), z2);
            out[2 * i] = from_f32<T>(s * __low2float(d));
            out[2 * i + 1] = from_f32<T>(s * __high2float(d));
        }
    }
}

struct CacheIo {
    CacheGeom g;
    const int64_t *slots;
    uint32_t tokens;
    int64_t k_token, k_head, v_token, v_head;   // strides in elements
    int k_vec, v_vec;
    unsigned *err;
};

// Lanes of a token's head, and tokens of a block of 256 threads.
template <int D>
struct IoCfg {
    static constexpr int LANES = D <= 64 ? 8 : 16, TOKENS = 256 / LANES;
};

// A block's head and a lane's eight channels of it; the block takes PER tokens a lane.
struct Lane {
    uint32_t head, c8, tok;   // tok: the first
    uint8_t *base;            // this head's block of page 0
};

template <int D, int PER>
__device__ __forceinline__ Lane io_lane(const CacheIo &a) {
    using F = IoCfg<D>;
    Lane l;
    const unsigned heads = static_cast<unsigned>(a.g.kv_heads), tile = blockIdx.x / heads;
    l.head = blockIdx.x - tile * heads;
    l.c8 = threadIdx.x % F::LANES;
    l.tok = tile * (F::TOKENS * PER) + threadIdx.x / F::LANES;
    l.base = a.g.data + l.head * a.g.block_bytes;
    return l;
}

// Where a token's head lies.
struct Cell {
    int64_t slot;
    bool live;                // a token of the list, with a slot in the cache
    uint8_t *blk;             // its page's block of this head
    uint32_t at;              // position in the page
};

__device__ __forceinline__ Cell io_cell(const CacheIo &a, const Lane &l, uint32_t tok) {
    Cell c;
    c.slot = tok < a.tokens ? a.slots[tok] : -1;
    const int64_t page = c.slot >> a.g.page_shift;
    c.live = c.slot >= 0 && page < a.g.pages;
    if (c.slot >= 0 && !c.live && l.c8 == 0) set_error(a.err, ERR_RANGE);
    c.blk = l.base + (c.live ? static_cast<uint64_t>(static_cast<uint32_t>(page)) * a.g.page_bytes : 0);
    c.at = static_cast<uint32_t>(c.slot) & ((1u << a.g.page_shift) - 1u);
    return c;
}

// Whether the token and the one LANES lanes away make a pair of neighbouring slots (even, odd): both lanes agree.
template <int LANES>
__device__ __forceinline__ bool paired(const Cell &c) {
    const int64_t other = __shfl_xor_sync(0xffffffffu, c.live ? c.slot : -1, LANES);
    return c.live && other >= 0 && other == (c.slot ^ 1) && ((threadIdx.x & LANES) != 0) == ((c.slot & 1) != 0);
}

template <int D, int PER, typename T>
__global__ void __launch_bounds__(256) k_cache_append(const CacheIo a, const T *K, const T *V) {
    constexpr int LANES = IoCfg<D>::LANES, TOKENS = IoCfg<D>::TOKENS, C = D / 32;
    const CacheGeom &g = a.g;
    const Lane l = io_lane<D, PER>(a);
    const bool inside = 8 * l.c8 < D, loads = 8 * l.c8 < static_cast<uint32_t>(g.dim);
    const T *kp = K + l.tok * a.k_token + l.head * a.k_head + 8 * l.c8, *vp = V + l.tok * a.v_token + l.head * a.v_head + 8 * l.c8;
#pragma unroll
    for (int n = 0; n < PER; ++n, kp += TOKENS * a.k_token, vp += TOKENS * a.v_token) {
        const Cell c = io_cell(a, l, l.tok + n * TOKENS);
        float k[8], v[8], k_lo = 0.0f, k_hi = 0.0f, v_lo = 0.0f, v_hi = 0.0f, odd_one = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = v[i] = 0.0f;
        if (c.live && loads) {
            load8(kp, a.k_vec != 0, k, k_lo, k_hi);
            load8(vp, a.v_vec != 0, v, v_lo, v_hi);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) odd_one = fmaf(k[i], 0.0f, fmaf(v[i], 0.0f, odd_one));   // NaN from a NaN or an infinity on
        bool bad = !(odd_one == 0.0f) || fmaxf(fmaxf(k_hi, -k_lo), fmaxf(v_hi, -v_lo)) > kCacheMaxAbs;
        const unsigned votes = __ballot_sync(0xffffffffu, bad) >> (threadIdx.x & 31 & ~(LANES - 1));
        bad = (votes & ((1u << LANES) - 1u)) != 0u;           // of the token's head
        if (bad) {
#pragma unroll
            for (int i = 0; i < 8; ++i) k[i] = v[i] = 0.0f;
            k_lo = k_hi = v_lo = v_hi = 0.0f;
            if (l.c8 == 0 && c.live) set_error(a.err, ERR_NUMERIC);
        }
        const int lanes = 1 << (g.group_shift - 3);           // of a group
        float ks, kz, vs, vz;
        group_grid<T>(k_lo, k_hi, lanes, ks, kz);
        group_grid<T>(v_lo, v_hi, lanes, vs, vz);
        // channels 8 c8 .. + 7 are word t = c8 % 4 of chunk w = c8 / 4; for values r = 2 t and 2 t + 1
        const uint32_t kw = codes8<T>(k, ks, kz, [](int i) { return 4 * (i >> 1) + 16 * (i & 1); });
        const uint32_t vw = codes8<T>(v, vs, vz, [](int i) { return 4 * i; });
        const bool pair = paired<LANES>(c);
        // of a pair the even token's lane writes the words of r = 2 t, the odd one's those of 2 t + 1
        const bool odd = (threadIdx.x & LANES) != 0;
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, odd ? vw & 0xffffu : vw >> 16, LANES);
        if (!c.live || !inside) continue;
        const uint32_t w = l.c8 >> 2, t = l.c8 & 3, j = c.at & 7;
        uint8_t *b8 = c.blk + (c.at >> 3) * (4 * D);          // the 8-token block's key codes
        *reinterpret_cast<uint32_t *>(b8 + 4 * ((4 * j + t) * C + w)) = kw;
        uint8_t *vb = b8 + g.v_off;
        if (pair) {
            const uint32_t word = odd ? theirs | (vw & 0xffff0000u) : (vw & 0xffffu) | theirs << 16;
            *reinterpret_cast<uint32_t *>(vb + 4 * ((4 * (2 * t + odd) + (j >> 1)) * C + w)) = word;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<uint16_t *>(vb + 4 * ((4 * (2 * t + h) + (j >> 1)) * C + w) + 2 * (j & 1)) =
                    static_cast<uint16_t>(vw >> (16 * h));
        }
        if ((l.c8 & (lanes - 1)) == 0) {
            const uint32_t word = c.at * g.groups + (l.c8 >> (g.group_shift - 3));
            reinterpret_cast<uint32_t *>(c.blk + g.kg_off)[word] =
                bad ? kBadKeyGrid : __float_as_uint(ks) | (__float_as_uint(kz) >> 16);
            reinterpret_cast<uint32_t *>(c.blk + g.vg_off)[word] =
                bad ? kBadValueGrid : __float_as_uint(vs) | (__float_as_uint(vz) >> 16);
        }
    }
}

template <int D, int PER, typename T>
__global__ void __launch_bounds__(256) k_cache_read(const CacheIo a, T *K, T *V) {
    constexpr int LANES = IoCfg<D>::LANES, TOKENS = IoCfg<D>::TOKENS, C = D / 32;
    const CacheGeom &g = a.g;
    const Lane l = io_lane<D, PER>(a);
    const bool inside = 8 * l.c8 < D;
    T *kto = K + l.tok * a.k_token + l.head * a.k_head + 8 * l.c8, *vto = V + l.tok * a.v_token + l.head * a.v_head + 8 * l.c8;
#pragma unroll
    for (int n = 0; n < PER; ++n, kto += TOKENS * a.k_token, vto += TOKENS * a.v_token) {
        const Cell c = io_cell(a, l, l.tok + n * TOKENS);
        const bool pair = paired<LANES>(c), odd = (threadIdx.x & LANES) != 0;
        const uint32_t w = l.c8 >> 2, t = l.c8 & 3, j = c.at & 7;
        uint32_t kw = 0u, vw = 0u, kg = 0u, vg = 0u;
        if (c.live && inside) {
            const uint8_t *b8 = c.blk + (c.at >> 3) * (4 * D);
            kw = *reinterpret_cast<const uint32_t *>(b8 + 4 * ((4 * j + t) * C + w));
            const uint8_t *vb = b8 + g.v_off;
            if (pair) {
                vw = *reinterpret_cast<const uint32_t *>(vb + 4 * ((4 * (2 * t + odd) + (j >> 1)) * C + w));
            } else {
                vw = *reinterpret_cast<const uint16_t *>(vb + 4 * (8 * t + (j >> 1)) * C + 4 * w + 2 * (j & 1));
                vw |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(vb + 4 * (8 * t + 4 + (j >> 1)) * C + 4 * w + 2 * (j & 1))) << 16;
            }
            const uint32_t word = c.at * g.groups + (l.c8 >> (g.group_shift - 3));
            kg = reinterpret_cast<const uint32_t *>(c.blk + g.kg_off)[word];
            vg = reinterpret_cast<const uint32_t *>(c.blk + g.vg_off)[word];
        }
        // of a pair the even token's lane read r = 2 t of both, the odd one's 2 t + 1: each hands over the other token's half
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, odd ? vw & 0xffffu : vw >> 16, LANES);
        if (pair) vw = odd ? theirs | (vw & 0xffff0000u) : (vw & 0xffffu) | theirs << 16;
        if (l.tok + n * TOKENS >= a.tokens || 8 * l.c8 >= static_cast<uint32_t>(g.dim)) continue;
        if (vg & 0x80000000u) vg = kBadKeyGrid;
        uint32_t kp[4], vp[4], vh[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kp[i] = (kw >> (4 * i)) & 0x000f000fu;            // channels 2 i, 2 i + 1
            vh[i] = (vw >> (4 * i)) & 0x000f000fu;            // channels i, i + 4
        }
        vp[0] = __byte_perm(vh[0], vh[1], 0x5410);
        vp[1] = __byte_perm(vh[2], vh[3], 0x5410);
        vp[2] = __byte_perm(vh[0], vh[1], 0x7632);
        vp[3] = __byte_perm(vh[2], vh[3], 0x7632);
        T k[8], v[8];
        values8(kp, kg, k);
        values8(vp, vg, v);
        if (K) store8(kto, a.k_vec != 0, k);
        if (V) store8(vto, a.v_vec != 0, v);
    }
}

template <int D, int PER, typename T, bool APPEND>
void launch_one(const CacheIo &io, void *K, void *V, cudaStream_t s) {
    const unsigned blocks = static_cast<unsigned>(ceil_div(io.tokens, IoCfg<D>::TOKENS * PER) * io.g.kv_heads);
    if constexpr (APPEND) k_cache_append<D, PER, T><<<blocks, 256, 0, s>>>(io, static_cast<const T *>(K), static_cast<const T *>(V));
    else k_cache_read<D, PER, T><<<blocks, 256, 0, s>>>(io, static_cast<T *>(K), static_cast<T *>(V));
}

template <int D, typename T, bool APPEND>
void launch_per(const CacheIo &io, void *K, void *V, cudaStream_t s) {
    // four tokens a lane where that still leaves the GPU full (its 1216 blocks of 256): what a lane works out once
    // is half of what a token costs it
    if (static_cast<int64_t>(io.tokens) * io.g.kv_heads >= int64_t{4} * 1216 * IoCfg<D>::TOKENS) launch_one<D, 4, T, APPEND>(io, K, V, s);
    else launch_one<D, 1, T, APPEND>(io, K, V, s);
}

template <typename T, bool APPEND>
cudaError_t launch_io(const CacheIo &io, void *K, void *V, cudaStream_t s) {
    if (io.g.D == 64) launch_per<64, T, APPEND>(io, K, V, s);
    else if (io.g.D == 96) launch_per<96, T, APPEND>(io, K, V, s);
    else launch_per<128, T, APPEND>(io, K, V, s);
    return cudaGetLastError();
}

template <bool APPEND>
qe_status launch_dtype(const CacheIo &io, void *K, void *V, qe_dtype dtype, cudaStream_t s) {
    const cudaError_t e = dtype == QE_F32 ? launch_io<float, APPEND>(io, K, V, s)
                          : dtype == QE_BF16 ? launch_io<__nv_bfloat16, APPEND>(io, K, V, s)
                                             : launch_io<__half, APPEND>(io, K, V, s);
    return e == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

bool wide_aligned(const void *p, int64_t s0, int64_t s1, int size) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && s0 % (16 / size) == 0 && s1 % (16 / size) == 0;
}

// Checks that the two calls share; `io` is filled but for the error word.
qe_status cache_io(const qe_cache *cache, const void *K, int64_t k_token, int64_t k_head, const void *V,
                   int64_t v_token, int64_t v_head, qe_dtype dtype, const int64_t *slots, int64_t tokens,
                   CacheIo *io) {
    if (tokens < 0 || (dtype != QE_F32 && dtype != QE_BF16 && dtype != QE_F16)) return QE_ERR_INVALID_ARG;
    const qe_status st = cache_geom(cache, &io->g);
    if (st != QE_OK) return st;
    if (tokens == 0) return QE_OK;
    if (tokens > 0x7fffffff || tokens > (int64_t{1} << 33) / io->g.kv_heads) return QE_ERR_INVALID_ARG;   // a grid's blocks
    const uintptr_t esize = dtype == QE_F32 ? 4 : 2;
    if (!slots || (reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || reinterpret_cast<uintptr_t>(K) % esize != 0 ||
        reinterpret_cast<uintptr_t>(V) % esize != 0)
        return QE_ERR_INVALID_ARG;
    const int size = dtype == QE_F32 ? 4 : 2;
    io->slots = slots;
    io->tokens = static_cast<uint32_t>(tokens);
    io->k_token = k_token;
    io->k_head = k_head;
    io->v_token = v_token;
    io->v_head = v_head;
    io->k_vec = wide_aligned(K, k_token, k_head, size);
    io->v_vec = wide_aligned(V, v_token, v_head, size);
    io->err = device_error_word();
    if (!io->err) return QE_ERR_CUDA;
    return QE_OK;
}

}  // namespace
}  // namespace qe

using namespace qe;

extern "C" {

qe_status qe_cache_size(int64_t pages, int page_size, int kv_heads, int head_dim, int group_size, size_t *bytes) {
    if (!bytes || pages < 1 || page_size < 1 || kv_heads < 1 || head_dim < 1 || group_size < 1) return QE_ERR_INVALID_ARG;
    if (page_size < 16 || page_size > 65536 || (page_size & (page_size - 1)) != 0) return QE_ERR_UNSUPPORTED;
    if (head_dim > 128 || head_dim % 8 != 0) return QE_ERR_UNSUPPORTED;
    const int D = cache_padded(head_dim);
    if ((group_size != 32 && group_size != 64 && group_size != 128) || D % group_size != 0) return QE_ERR_UNSUPPORTED;
    if (kv_heads > 65535 || pages > 0x7fffffff) return QE_ERR_INVALID_ARG;
    const uint64_t block = static_cast<uint64_t>(D + 8 * (D / group_size)) * static_cast<uint64_t>(page_size);
    if (block * kv_heads >= (static_cast<uint64_t>(1) << 31)) return QE_ERR_UNSUPPORTED;
    *bytes = static_cast<size_t>(static_cast<uint64_t>(pages) * kv_heads * block);
    return QE_OK;
}

qe_status qe_cache_append(const qe_cache *cache, const void *K, int64_t k_token, int64_t k_head, const void *V,
                          int64_t v_token, int64_t v_head, qe_dtype dtype, const int64_t *slots, int64_t tokens,
                          qe_stream_t stream) {
    CacheIo io{};
    if (tokens > 0 && (!K || !V)) return QE_ERR_INVALID_ARG;
    const qe_status st = cache_io(cache, K, k_token, k_head, V, v_token, v_head, dtype, slots, tokens, &io);
    if (st != QE_OK || tokens == 0) return st;
    return launch_dtype<true>(io, const_cast<void *>(K), const_cast<void *>(V), dtype, reinterpret_cast<cudaStream_t>(stream));
}

qe_status qe_cache_read(const qe_cache *cache, const int64_t *slots, int64_t tokens, void *K, int64_t k_token,
                        int64_t k_head, void *V, int64_t v_token, int64_t v_head, qe_dtype dtype, qe_stream_t stream) {
    CacheIo io{};
    if (tokens > 0 && !K && !V) return QE_ERR_INVALID_ARG;
    const qe_status st = cache_io(cache, K, k_token, k_head, V, v_token, v_head, dtype, slots, tokens, &io);
    if (st != QE_OK || tokens == 0) return st;
    return launch_dtype<false>(io, K, V, dtype, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
