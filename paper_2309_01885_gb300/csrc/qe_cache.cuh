// The 4-bit key/value cache: its geometry and the layout of its bytes.
//
// Keys and values are codes on uniform grids x^ = s (c - z), one grid for each
// token, kv head and group of G channels: the per-row grid of the layer
// quantizer (0 in range, integer z, ties to even), with the scale rounded to
// bf16 before z and the codes are taken from it, so that a grid costs one
// 32-bit word and the codes still are the nearest levels of the stored grid.
//
// Channels are padded to D = 64, 96 or 128 (C = D / 32 chunks).  A page of P
// tokens holds one block per kv head: key codes (P D / 2 bytes), value codes
// (the same), key grids (P words per group), value grids.  Codes are 32-bit
// words in 8-token blocks of 32 lanes x C words, so that a warp reads a block
// as one contiguous access and lane l finds in its C words what the fragments
// of a 16-token matrix instruction want from it:
//   keys   lane 4 j + t, word w: token j, channels 32 w + 8 t + 2 p + h at bit
//          4 p + 16 h: masking with 0x000f000f << 4 p leaves a pair of channels;
//   values lane 4 r + t, word w: channels 32 w + 4 r + i of tokens 2 t + h at bit
//          4 i + 16 h: the same masks leave one channel of a pair of tokens, and
//          a token owns whole 16-bit halves (a token is written without reading).
#pragma once

#include "../../include/qe.h"
#include "qe_common.cuh"

namespace qe {

constexpr uint32_t kBadKeyGrid = 0x7FC00000u;     // scale NaN: every row that sees the token becomes NaN
constexpr uint32_t kBadValueGrid = 0x80000000u;   // scale -0: adds nothing to a row that does not see it, reads back as NaN
constexpr float kCacheMaxAbs = 8.5070592e37f;     // 2^126: larger magnitudes count as non-finite (hi - lo stays finite)

// What the kernels need of a qe_cache.
struct CacheGeom {
    uint8_t *data;
    int64_t pages;
    uint32_t block_bytes;     // one page of one kv head
    uint32_t page_bytes;      // one page: offsets inside it fit in 32 bits
    uint32_t v_off, kg_off, vg_off;   // parts of a block: value codes, key grids, value grids
    int page_shift;           // log2(page_size)
    int kv_heads;
    int dim;                  // channels of a head
    int D;                    // padded to 64, 96 or 128
    int group_shift;          // log2(group_size)
    int groups;               // D / group_size
};

__host__ __device__ inline int cache_padded(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }

// Checks a qe_cache and fills the geometry; QE_ERR_INVALID_ARG / QE_ERR_UNSUPPORTED otherwise.
qe_status cache_geom(const qe_cache *cache, CacheGeom *g);

}  // namespace qe
