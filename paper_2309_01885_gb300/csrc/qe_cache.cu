// Writing the 4-bit key/value cache and reading it back (layout: qe_cache.cuh).
//
// Both kernels give four channels of a token's head to a lane: a group of G
// channels is G / 4 neighbouring lanes, whose minimum and maximum meet in
// shuffles, and a lane's four value codes are one 16-bit half of the layout.
// They move 2 + 0.5 + 4 / G bytes per 16-bit channel and are bound by HBM.
#include <cuda_fp16.h>

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
    g->block_bytes = static_cast<int64_t>(g->D + 8 * g->groups) * c->page_size;
    return QE_OK;
}

namespace {

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return static_cast<float>(v); }

// Four neighbouring channels; `vec`: the address is aligned to them.
template <typename T>
__device__ __forceinline__ void load4(const T *p, bool vec, int n, float (&v)[4]) {
    if (vec && n >= 4) {
        if constexpr (sizeof(T) == 4) {
            const float4 t = *reinterpret_cast<const float4 *>(p);
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
            union { uint2 u; T e[4]; } t;
            t.u = *reinterpret_cast<const uint2 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = to_f32(t.e[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <typename T>
__device__ __forceinline__ void store4(T *p, bool vec, int n, const float (&v)[4]) {
    if (vec && n >= 4) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            union { uint2 u; T e[4]; } t;
#pragma unroll
            for (int i = 0; i < 4; ++i) t.e[i] = from_f32<T>(v[i]);
            *reinterpret_cast<uint2 *>(p) = t.u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

// The grid of a group whose channels lie in 2^steps neighbouring lanes (four each).
__device__ __forceinline__ void group_grid(const float (&x)[4], int lanes, float &s, float &z) {
    float lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    float hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    for (int o = 1; o < lanes; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    lo = fminf(lo, 0.0f);
    hi = fmaxf(hi, 0.0f);
    const float r = __fdiv_rn(__fsub_rn(hi, lo), 15.0f);
    s = fmaxf(__bfloat162float(__float2bfloat16_rn(r)), 1.17549435e-38f);
    z = rintf(__fdiv_rn(fabsf(lo), s));
}

__device__ __forceinline__ uint32_t nearest_code(float x, float s, float z) {
    const float c = rintf(__fdiv_rn(x, s)) + z;
    return static_cast<uint32_t>(fminf(fmaxf(c, 0.0f), 15.0f));
}

struct CacheIo {
    CacheGeom g;
    const int64_t *slots;
    int64_t tokens;
    int64_t k_token, k_head, v_token, v_head;   // strides in elements
    int k_vec, v_vec;
    unsigned *err;
};

// One item = one token's kv head; D / 4 lanes of a warp (half a warp for D = 64).
template <typename T>
__global__ void __launch_bounds__(256) k_cache_append(const CacheIo a, const T *K, const T *V) {
    const CacheGeom &g = a.g;
    const int lane = threadIdx.x & 31;
    const int per = g.D == 64 ? 2 : 1;                       // items of a warp
    const int sub = per == 2 ? lane >> 4 : 0;
    const int l = per == 2 ? lane & 15 : lane;               // quad of channels 4 l .. 4 l + 3
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5;
    const int64_t items = a.tokens * g.kv_heads;
    const int64_t item = warp * per + sub;
    if (warp * per >= items) return;                         // uniform in the warp
    const int64_t tok = item / g.kv_heads;
    const int head = static_cast<int>(item - tok * g.kv_heads);
    bool live = item < items && 4 * l < g.D;
    const int64_t slot = item < items ? a.slots[tok] : -1;
    const int64_t page = slot >> g.page_shift;
    if (slot < 0) live = false;
    else if (page >= g.pages) {
        live = false;
        if (l == 0) set_error(a.err, ERR_RANGE);
    }
    float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (live && 4 * l < g.dim) {
        load4(K + tok * a.k_token + head * a.k_head + 4 * l, a.k_vec != 0, g.dim - 4 * l, k);
        load4(V + tok * a.v_token + head * a.v_head + 4 * l, a.v_vec != 0, g.dim - 4 * l, v);
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        bad = bad || !(fabsf(k[i]) <= kCacheMaxAbs) || !(fabsf(v[i]) <= kCacheMaxAbs);
    const unsigned votes = __ballot_sync(0xffffffffu, bad);
    bad = ((per == 2 ? (votes >> (16 * sub)) & 0xffffu : votes) != 0u);
    if (bad) {
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = v[i] = 0.0f;
        if (l == 0 && live) set_error(a.err, ERR_NUMERIC);
    }
    const int lanes = 1 << (g.group_shift - 2);              // lanes of a group
    float ks, kz, vs, vz;
    group_grid(k, lanes, ks, kz);
    group_grid(v, lanes, vs, vz);
    uint32_t kw = 0u, vw = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        kw |= nearest_code(k[i], ks, kz) << (4 * ((i >> 1) + 2 * (l & 1)) + 16 * (i & 1));
        vw |= nearest_code(v[i], vs, vz) << (4 * i);
    }
    kw |= __shfl_xor_sync(0xffffffffu, kw, 1);
    if (!live) return;
    const int C = g.D >> 5, w = l >> 3;
    const int64_t at = slot & ((static_cast<int64_t>(1) << g.page_shift) - 1);
    uint8_t *blk = g.data + (page * g.kv_heads + head) * g.block_bytes;
    const int64_t b8 = (at >> 3) * (4 * g.D);                // bytes of the 8-token blocks before
    const int j = static_cast<int>(at & 7);
    if ((l & 1) == 0)
        *reinterpret_cast<uint32_t *>(blk + b8 + 4 * ((4 * j + ((l & 7) >> 1)) * C + w)) = kw;
    *reinterpret_cast<uint16_t *>(blk + cache_v_off(g) + b8 + 4 * ((4 * (l & 7) + (j >> 1)) * C + w) + 2 * (j & 1)) =
        static_cast<uint16_t>(vw);
    if ((l & (lanes - 1)) == 0) {
        const int64_t word = at * g.groups + (l >> (g.group_shift - 2));
        reinterpret_cast<uint32_t *>(blk + cache_kg_off(g))[word] =
            bad ? kBadKeyGrid : __float_as_uint(ks) | (__float_as_uint(kz) >> 16);
        reinterpret_cast<uint32_t *>(blk + cache_vg_off(g))[word] =
            bad ? kBadValueGrid : __float_as_uint(vs) | (__float_as_uint(vz) >> 16);
    }
}

__device__ __forceinline__ float grid_scale(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float grid_zero(uint32_t w) { return __uint_as_float(w << 16); }

template <typename T>
__global__ void __launch_bounds__(256) k_cache_read(const CacheIo a, T *K, T *V) {
    const CacheGeom &g = a.g;
    const int lane = threadIdx.x & 31;
    const int per = g.D == 64 ? 2 : 1;
    const int l = per == 2 ? lane & 15 : lane;
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5;
    const int64_t item = warp * per + (per == 2 ? lane >> 4 : 0);
    if (item >= a.tokens * g.kv_heads || 4 * l >= g.dim) return;
    const int64_t tok = item / g.kv_heads;
    const int head = static_cast<int>(item - tok * g.kv_heads);
    const int64_t slot = a.slots[tok];
    const int64_t page = slot >> g.page_shift;
    float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && page >= g.pages) {
        if (l == 0) set_error(a.err, ERR_RANGE);
    } else if (slot >= 0) {
        const int C = g.D >> 5, w = l >> 3;
        const int64_t at = slot & ((static_cast<int64_t>(1) << g.page_shift) - 1);
        const uint8_t *blk = g.data + (page * g.kv_heads + head) * g.block_bytes;
        const int64_t b8 = (at >> 3) * (4 * g.D);
        const int j = static_cast<int>(at & 7);
        const uint32_t kw =
            *reinterpret_cast<const uint32_t *>(blk + b8 + 4 * ((4 * j + ((l & 7) >> 1)) * C + w)) >> (8 * (l & 1));
        const uint32_t vw = *reinterpret_cast<const uint16_t *>(blk + cache_v_off(g) + b8 +
                                                                4 * ((4 * (l & 7) + (j >> 1)) * C + w) + 2 * (j & 1));
        const int64_t word = at * g.groups + (l >> (g.group_shift - 2));
        const uint32_t kg = reinterpret_cast<const uint32_t *>(blk + cache_kg_off(g))[word];
        uint32_t vg = reinterpret_cast<const uint32_t *>(blk + cache_vg_off(g))[word];
        if (vg & 0x80000000u) vg = kBadKeyGrid;
        const float ks = grid_scale(kg), kz = grid_zero(kg), vs = grid_scale(vg), vz = grid_zero(vg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            k[i] = ks * (static_cast<float>((kw >> (4 * (i >> 1) + 16 * (i & 1))) & 15u) - kz);
            v[i] = vs * (static_cast<float>((vw >> (4 * i)) & 15u) - vz);
        }
    }
    if (K) store4(K + tok * a.k_token + head * a.k_head + 4 * l, a.k_vec != 0, g.dim - 4 * l, k);
    if (V) store4(V + tok * a.v_token + head * a.v_head + 4 * l, a.v_vec != 0, g.dim - 4 * l, v);
}

bool quads_aligned(const void *p, int64_t s0, int64_t s1, int size) {
    return (reinterpret_cast<uintptr_t>(p) % (4 * size)) == 0 && s0 % 4 == 0 && s1 % 4 == 0;
}

// Checks that the two calls share; `io` is filled but for the error word.
qe_status cache_io(const qe_cache *cache, const void *K, int64_t k_token, int64_t k_head, const void *V,
                   int64_t v_token, int64_t v_head, qe_dtype dtype, const int64_t *slots, int64_t tokens,
                   CacheIo *io) {
    if (tokens < 0 || (dtype != QE_F32 && dtype != QE_BF16 && dtype != QE_F16)) return QE_ERR_INVALID_ARG;
    const qe_status st = cache_geom(cache, &io->g);
    if (st != QE_OK) return st;
    if (tokens == 0) return QE_OK;
    if (tokens > (int64_t{1} << 33) / io->g.kv_heads) return QE_ERR_INVALID_ARG;   // a grid's blocks
    const uintptr_t esize = dtype == QE_F32 ? 4 : 2;
    if (!slots || (reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || reinterpret_cast<uintptr_t>(K) % esize != 0 ||
        reinterpret_cast<uintptr_t>(V) % esize != 0)
        return QE_ERR_INVALID_ARG;
    const int size = dtype == QE_F32 ? 4 : 2;
    io->slots = slots;
    io->tokens = tokens;
    io->k_token = k_token;
    io->k_head = k_head;
    io->v_token = v_token;
    io->v_head = v_head;
    io->k_vec = quads_aligned(K, k_token, k_head, size);
    io->v_vec = quads_aligned(V, v_token, v_head, size);
    io->err = device_error_word();
    if (!io->err) return QE_ERR_CUDA;
    return QE_OK;
}

// Blocks of 8 warps over the items.
unsigned item_blocks(const CacheIo &io) {
    const int64_t warps = ceil_div(io.tokens * io.g.kv_heads, io.g.D == 64 ? 2 : 1);
    return static_cast<unsigned>(ceil_div(warps, 8));
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
    if (static_cast<uint64_t>(pages) > (static_cast<uint64_t>(1) << 62) / (block * kv_heads)) return QE_ERR_INVALID_ARG;
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
    const unsigned blocks = item_blocks(io);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == QE_F32)
        k_cache_append<float><<<blocks, 256, 0, s>>>(io, static_cast<const float *>(K), static_cast<const float *>(V));
    else if (dtype == QE_BF16)
        k_cache_append<__nv_bfloat16><<<blocks, 256, 0, s>>>(io, static_cast<const __nv_bfloat16 *>(K),
                                                             static_cast<const __nv_bfloat16 *>(V));
    else
        k_cache_append<__half><<<blocks, 256, 0, s>>>(io, static_cast<const __half *>(K), static_cast<const __half *>(V));
    return cudaGetLastError() == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

qe_status qe_cache_read(const qe_cache *cache, const int64_t *slots, int64_t tokens, void *K, int64_t k_token,
                        int64_t k_head, void *V, int64_t v_token, int64_t v_head, qe_dtype dtype, qe_stream_t stream) {
    CacheIo io{};
    if (tokens > 0 && !K && !V) return QE_ERR_INVALID_ARG;
    const qe_status st = cache_io(cache, K, k_token, k_head, V, v_token, v_head, dtype, slots, tokens, &io);
    if (st != QE_OK || tokens == 0) return st;
    const unsigned blocks = item_blocks(io);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == QE_F32)
        k_cache_read<float><<<blocks, 256, 0, s>>>(io, static_cast<float *>(K), static_cast<float *>(V));
    else if (dtype == QE_BF16)
        k_cache_read<__nv_bfloat16><<<blocks, 256, 0, s>>>(io, static_cast<__nv_bfloat16 *>(K),
                                                           static_cast<__nv_bfloat16 *>(V));
    else
        k_cache_read<__half><<<blocks, 256, 0, s>>>(io, static_cast<__half *>(K), static_cast<__half *>(V));
    return cudaGetLastError() == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

}  // extern "C"
