// Products with a quantized layer: the entry points, and laying a layer out (layout:
// qe_linear.cuh; kernels: qe_linear_rows.cuh for a few rows, qe_linear_tiles.cuh for many).
#include "qe_internal.h"
#include "qe_linear.cuh"

namespace qe {
namespace {

// Where a pair's code stands: bit j of column e (0, 1) of pair p of half h of chunk c.
template <int B>
__device__ __forceinline__ void enter(uint32_t (&w)[B], int c, int h, int p, int e, uint32_t code) {
    if constexpr (B == 2) w[c] |= code << (2 * (4 * h + p) + 16 * e);
    if constexpr (B == 4) w[2 * c + h] |= code << (4 * p + 16 * e);
    if constexpr (B == 8) w[4 * c + 2 * h + (p >> 1)] |= code << (8 * (p & 1) + 16 * e);
    if constexpr (B == 3) {
        const int i = 8 * c + 4 * h + p;
        if (i < 15) {
            w[i / 5] |= code << (3 * (i % 5) + 16 * e);
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j) w[j] |= (code >> j & 1u) << (15 + 16 * e);
        }
    }
}

// A warp lays out a unit.
template <int B>
__global__ void __launch_bounds__(256) k_linear_codes(const LinearGeom g, uint8_t *to, const uint8_t *codes, int64_t ldc, uint32_t mask) {
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (unit >= static_cast<int64_t>(g.row_tiles) * g.units) return;
    const int64_t tile = unit / g.units, col = (unit - tile * g.units) * kUnitCols;
    const int lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    uint32_t w[B];
#pragma unroll
    for (int j = 0; j < B; ++j) w[j] = 0u;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t i = tile * kTileRows + r + 8 * h, k = col + 32 * c + 2 * t;
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int e = 0; e < 2; ++e) enter<B>(w, c, h, p, e, i < g.q && k + 8 * p + e < g.p ? codes[i * ldc + k + 8 * p + e] & mask : 0u);
        }
    uint32_t *out = reinterpret_cast<uint32_t *>(to + unit * (128 * B));
#pragma unroll
    for (int j = 0; j < B; ++j) out[unit_word(B, lane, j)] = w[j];
}

__global__ void __launch_bounds__(256) k_linear_grids(const LinearGeom g, float *scales, uint8_t *zeros, const float *from_s, const float *from_z,
                                                      float top, unsigned *err) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    // (of an odd number of row tiles the last pair's second one is written too)
    if (n >= static_cast<int64_t>(g.row_tiles + (g.row_tiles & 1)) * g.groups * kTileRows) return;
    const int64_t tile = n / (g.groups * kTileRows), i = tile * kTileRows + n % kTileRows, grp = n / kTileRows % g.groups;
    float s = 0.0f, z = 0.0f;
    if (i < g.q) {
        s = from_s[i * g.groups + grp];
        z = from_z[i * g.groups + grp];
        if (!(fabsf(s) <= 3.40282347e38f) || !(z >= 0.0f && z <= top) || z != rintf(z)) {
            s = __uint_as_float(0x7FC00000u);
            z = 0.0f;
            set_error(err, ERR_NUMERIC);
        }
    }
    if (tile < g.row_tiles) scales[n] = s;
    const int row = static_cast<int>(n % kTileRows);
    zeros[((tile >> 1) * g.groups + grp) * 32 + 4 * (row & 7) + 2 * (tile & 1) + (row >> 3)] = static_cast<uint8_t>(z);
}

// Rows of x at a pitch of whole 16 bytes, for calls whose own rows are not aligned so.
__global__ void __launch_bounds__(256) k_linear_align(const uint16_t *x, int64_t ldx, int64_t rows, int64_t p, uint16_t *to, int64_t ld) {
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y)
        for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < p; k += static_cast<int64_t>(gridDim.x) * 256)
            to[m * ld + k] = x[m * ldx + k];
}

int64_t code_bytes(const LinearGeom &g) { return static_cast<int64_t>(g.row_tiles) * g.units * (128 * g.bits); }
int64_t grid_count(const LinearGeom &g) { return static_cast<int64_t>(g.row_tiles) * g.groups * kTileRows; }
int64_t zero_count(const LinearGeom &g) { return static_cast<int64_t>(g.row_tiles + (g.row_tiles & 1)) * g.groups * kTileRows; }

qe_status shape(int64_t q, int64_t p, int bits, int64_t group_size, LinearGeom *g, size_t *bytes) {
    if (q < 1 || p < 1 || q > (1 << 24) || p > (1 << 24) || bits < 2 || bits > 8 || group_size < 0) return QE_ERR_INVALID_ARG;
    const bool grouped = group_size > 0 && group_size < p;
    if (grouped && group_size % kUnitCols != 0) return QE_ERR_UNSUPPORTED;
    g->q = q;
    g->p = p;
    g->bits = stored_bits(bits);
    g->units = static_cast<int>(ceil_div(p, kUnitCols));
    g->row_tiles = static_cast<int>(ceil_div(q, kTileRows));
    g->groups = grouped ? static_cast<int>(ceil_div(p, group_size)) : 1;
    g->group_units = grouped ? static_cast<int>(group_size / kUnitCols) : g->units;
    *bytes = static_cast<size_t>(round_up(code_bytes(*g), 256) + round_up(4 * grid_count(*g), 256) + round_up(zero_count(*g), 256));
    return QE_OK;
}

}  // namespace

qe_status linear_geom(const qe_layer *layer, LinearGeom *g) {
    if (!layer || !layer->data || (reinterpret_cast<uintptr_t>(layer->data) & 255u) != 0) return QE_ERR_INVALID_ARG;
    size_t need = 0;
    const qe_status st = shape(layer->q, layer->p, layer->bits, layer->group_size, g, &need);
    if (st != QE_OK) return st;
    if (layer->bytes < need) return QE_ERR_INVALID_ARG;
    uint8_t *at = static_cast<uint8_t *>(layer->data);
    g->codes = at;
    at += round_up(code_bytes(*g), 256);
    g->scales = reinterpret_cast<const float *>(at);
    g->zeros = reinterpret_cast<const uint32_t *>(at + round_up(4 * grid_count(*g), 256));
    return QE_OK;
}

int linear_sms() {
    static std::atomic<int> known[64];                   // by device; 0: not asked yet
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && dev < 64 && (v = known[dev].load(std::memory_order_relaxed)) > 0) return v;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v < 1) {
        cudaGetLastError();
        return 152;
    }
    if (dev < 64) known[dev].store(v, std::memory_order_relaxed);
    return v;
}

RowsPlan rows_plan(const LinearArgs &a) {
    const int nt = static_cast<int>(a.rows <= 8 ? 1 : a.rows <= 16 ? 2 : a.rows <= 24 ? 3 : 4);
    RowsPlan best{1, 1};
    int64_t least = -1;
    for (int tiles = a.g.bits == 8 || nt > 1 ? 1 : 2; tiles >= 1; --tiles) {
        const int64_t groups = ceil_div(a.g.row_tiles, 8 * tiles) * ceil_div(a.rows, 8 * nt);
        for (int ranks = 1; ranks <= 8; ++ranks) {
            // An SM's time goes by the units it turns: its CTAs', each with what a CTA costs besides; one CTA alone leaves
            // pauses.  Measured (us, 4 bits, one / two row tiles a warp): 5 x 14848 x 59392 1 rank 176 / 283, 2 125 / 152 (116
            // CTAs), 4 121 / 118, 5 119 / 98 (290), 6 102 / 115, 7 107 / 102, 8 109 / 115; 1 x 4096 x 11008 39 / 66, 27 / 37,
            // 18 / 25, 18 / 20, 16 / 20, 16 / 23, 16 / 20; 24 x 11008 x 4096 in groups of 128 (one row tile) 39, 27 with 2,
            // 23 with 3 (258), 29 with 4 and more.
            const int64_t an_sm = ceil_div(groups * ranks, linear_sms());
            const int64_t cost = an_sm * (tiles * ceil_div(a.g.units, ranks) + 10) * (an_sm == 1 ? 4 : 3);
            if (least < 0 || cost < least) {
                least = cost;
                best = RowsPlan{tiles, ranks};
            }
        }
    }
    return best;
}

TilesPlan tiles_plan(const LinearArgs &a) {
    const int64_t outs = ceil_div(a.g.q, 128), sms = linear_sms();
    TilesPlan best{64, 64, 1};
    if (a.rows > 64) {
        // As many rows a tile as the rounds over the SMs ask for; a tile costs its rows and some 32 more, which it takes to
        // begin and to leave.  Measured (us, 4 bits, tiles of 128 / 160 / 192 / 224 / 256 rows): 4095 x 4096 x 11008 324 / 285 /
        // 248 / 215 / 229, 2048 x 4096 x 4096 88 / 74 / 74 / 68 / 59, 4095 x 14848 x 4096 516 / 434 / 375 / 338 / 311.
        const int room = a.rows <= 128 ? 128 : a.g.bits == 8 ? 224 : 256;   // (8 bits' codes take shared memory from x)
        int64_t least = -1;
        for (int rows = room; rows >= room / 2; rows -= 32) {
            const int64_t cost = ceil_div(outs * ceil_div(a.rows, rows), sms) * (rows + 32);
            if (least < 0 || cost < least) {
                least = cost;
                best = TilesPlan{room, rows, 1};
            }
        }
    }
    const int64_t tiles = outs * ceil_div(a.rows, best.rows);
    // A cluster shares a tile's columns out while one of twice its size finds SMs.  Measured (us, 1 / 2 / 4 / 8 CTAs): 64 x 4096 x
    // 4096 (32 tiles) 25 / 18 / 14 / 27, 128 x 4096 x 4096 (64) 29 / 18 / 25 / 45, 300 x 4096 x 4096 (96) 33 / 33 / 37 / 68.
    while (best.ranks < 8 && tiles * best.ranks * 2 <= sms && a.g.units >= 8 * best.ranks) best.ranks *= 2;
    return best;
}

namespace {

cudaError_t launch_rows(const LinearArgs &a, cudaStream_t s) {
    switch (a.g.bits) {
        case 2: return launch_linear_rows_2(a, s);
        case 3: return launch_linear_rows_3(a, s);
        case 4: return launch_linear_rows_4(a, s);
        default: return launch_linear_rows_8(a, s);
    }
}

cudaError_t launch_tiles(const LinearArgs &a, cudaStream_t s) {
    switch (a.g.bits) {
        case 2: return launch_linear_tiles_2(a, s);
        case 3: return launch_linear_tiles_3(a, s);
        case 4: return launch_linear_tiles_4(a, s);
        default: return launch_linear_tiles_8(a, s);
    }
}

// Rows of x up to which the few-rows kernel takes a call.  Measured (us, few rows / tiles): 4 bits, 4096 x 4096 9 to 32 rows 12 / 14,
// 64 16 / 14, 4096 x 11008 32 rows 20 / 20, 14848 x 14848 9 rows 45 / 63, 32 59 / 66, 14848 x 59392 24 rows 156 / 231, 32 180 / 231,
// 64 346 / 231; 8 bits, 4096 x 4096 9 to 32 rows 16 / 16, 11008 x 4096 32 rows 27 / 33, 14848 x 14848 80 / 94; groups of 128, 32 rows of
// 11008 x 4096, 4 bits 25 / 31, 8 bits 33 / 41, of 14848 x 14848 74 / 88 and 104 / 121.  (Short layers with groups take a little longer
// this way: 4096 x 4096 in groups of 128, 17 rows, 4 bits 16 / 14, 8 bits 20 / 18.)
constexpr int kFewRows = 32;

}  // namespace

}  // namespace qe

using namespace qe;

namespace {

bool halves(qe_dtype d) { return d == QE_BF16 || d == QE_F16; }

int64_t aligned_ld(int64_t p) { return round_up(p, 8); }

}  // namespace

extern "C" {

qe_status qe_linear_size(int64_t q, int64_t p, int bits, int64_t group_size, size_t *bytes) {
    LinearGeom g;
    if (!bytes) return QE_ERR_INVALID_ARG;
    return shape(q, p, bits, group_size, &g, bytes);
}

qe_status qe_linear_pack(const qe_layer *layer, const uint8_t *codes, int64_t ldc, const float *scales, const float *zeros, qe_stream_t stream) {
    LinearGeom g;
    const qe_status st = linear_geom(layer, &g);
    if (st != QE_OK) return st;
    if (!codes || !scales || !zeros || ldc < g.p || ((reinterpret_cast<uintptr_t>(scales) | reinterpret_cast<uintptr_t>(zeros)) & 3u) != 0)
        return QE_ERR_INVALID_ARG;
    unsigned *err = device_error_word();
    if (!err) return QE_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint8_t *to = static_cast<uint8_t *>(layer->data);
    const unsigned blocks = static_cast<unsigned>(ceil_div(static_cast<int64_t>(g.row_tiles) * g.units, 8));
    const uint32_t mask = (1u << layer->bits) - 1u;
    if (g.bits == 2) k_linear_codes<2><<<blocks, 256, 0, s>>>(g, to, codes, ldc, mask);
    else if (g.bits == 3) k_linear_codes<3><<<blocks, 256, 0, s>>>(g, to, codes, ldc, mask);
    else if (g.bits == 4) k_linear_codes<4><<<blocks, 256, 0, s>>>(g, to, codes, ldc, mask);
    else k_linear_codes<8><<<blocks, 256, 0, s>>>(g, to, codes, ldc, mask);
    if (cudaGetLastError() != cudaSuccess) return QE_ERR_CUDA;
    k_linear_grids<<<static_cast<unsigned>(ceil_div(zero_count(g), 256)), 256, 0, s>>>(
        g, const_cast<float *>(g.scales), reinterpret_cast<uint8_t *>(const_cast<uint32_t *>(g.zeros)), scales, zeros, static_cast<float>(mask), err);
    return cudaGetLastError() == cudaSuccess ? QE_OK : QE_ERR_CUDA;
}

qe_status qe_linear_workspace(const qe_layer *layer, int64_t rows, size_t *bytes) {
    LinearGeom g;
    if (!bytes || !layer || rows < 0 || rows > 0x7fffffff) return QE_ERR_INVALID_ARG;
    const qe_status st = shape(layer->q, layer->p, layer->bits, layer->group_size, &g, bytes);
    if (st != QE_OK) return st;
    *bytes = static_cast<size_t>(2 * rows * aligned_ld(g.p));
    return QE_OK;
}

qe_status qe_linear(const qe_layer *layer, const qe_product *pr, void *workspace, size_t workspace_bytes, qe_stream_t stream) {
    LinearArgs a{};
    const qe_status st = linear_geom(layer, &a.g);
    if (st != QE_OK) return st;
    if (!pr || pr->rows < 0 || pr->rows > 0x7fffffff || pr->act < QE_ACT_NONE || pr->act > QE_ACT_SILU) return QE_ERR_INVALID_ARG;
    if (!halves(pr->dtype)) return pr->dtype == QE_F32 ? QE_ERR_UNSUPPORTED : QE_ERR_INVALID_ARG;
    if (pr->bias && pr->bias_dtype != QE_F32 && !halves(pr->bias_dtype)) return QE_ERR_INVALID_ARG;
    if (pr->rows == 0) return QE_OK;
    if (!pr->X || !pr->Y || pr->ldx < a.g.p || pr->ldy < a.g.q || (pr->residual && pr->ldr < a.g.q)) return QE_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(pr->X) | reinterpret_cast<uintptr_t>(pr->Y) | reinterpret_cast<uintptr_t>(pr->residual)) & 1u) != 0 ||
        (reinterpret_cast<uintptr_t>(pr->bias) & (pr->bias_dtype == QE_F32 ? 3u : 1u)) != 0 || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
        return QE_ERR_INVALID_ARG;
    a.x = pr->X;
    a.ldx = pr->ldx;
    a.rows = pr->rows;
    a.half = pr->dtype == QE_F16;
    a.x_vec = (reinterpret_cast<uintptr_t>(pr->X) & 15u) == 0 && pr->ldx % 8 == 0;
    a.bias = pr->bias;
    a.bias_dtype = pr->bias_dtype;
    a.act = pr->act;
    a.residual = pr->residual;
    a.ldr = pr->ldr;
    a.y = pr->Y;
    a.ldy = pr->ldy;
    a.err = device_error_word();
    if (!a.err) return QE_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    void *own = nullptr;
    if (pr->rows <= kFewRows) {
        e = launch_rows(a, s);
    } else {
        if (!a.x_vec) {                                   // TMA wants rows that begin on 16 bytes
            const int64_t ld = aligned_ld(a.g.p);
            const size_t need = static_cast<size_t>(2 * pr->rows * ld);
            if (workspace && workspace_bytes < need) return QE_ERR_OOM;
            if (!workspace && cudaMallocAsync(&own, need, s) != cudaSuccess) {
                cudaGetLastError();
                return QE_ERR_OOM;
            }
            uint16_t *to = static_cast<uint16_t *>(workspace ? workspace : own);
            const dim3 grid(static_cast<unsigned>(ceil_div(a.g.p, 2048)), static_cast<unsigned>(pr->rows < 65535 ? pr->rows : 65535));
            k_linear_align<<<grid, 256, 0, s>>>(static_cast<const uint16_t *>(a.x), a.ldx, a.rows, a.g.p, to, ld);
            e = cudaGetLastError();
            a.x = to;
            a.ldx = ld;
        }
        if (e == cudaSuccess) e = launch_tiles(a, s);
    }
    if (own) cudaFreeAsync(own, s);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return QE_ERR_CUDA;
    }
    return QE_OK;
}

}  // extern "C"
