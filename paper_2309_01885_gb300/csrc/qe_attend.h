// Arguments and launchers of attention over the 4-bit key/value cache.
#pragma once

#include "qe_cache.cuh"

namespace qe {

struct AttendArgs {
    CacheGeom g;
    const int32_t *q_start, *kv_len, *table;
    int64_t table_ld;
    int64_t rows;             // query rows in all
    int64_t seqs;
    int64_t max_q;
    int q_heads, per_kv;      // query heads, query heads of a kv head
    int causal;
    int64_t window;           // 0 = none
    float scale2;             // softmax scale x log2 e
    const void *Q;
    void *out;
    int64_t q_row, q_head, o_row, o_head;   // strides in elements
    int half;                 // 1 = fp16, 0 = bf16
    int q_vec;                // 16-byte loads of Q are aligned
    float *lse;               // [rows][q_heads], natural log, or NULL
    int splits;               // pieces of a sequence's visible tokens
    int64_t min_tokens;       // a piece is not shorter than this
    float *part;              // splits > 1: [splits][rows][q_heads][dim] and, after them, [splits][rows][q_heads] (m, l)
    unsigned *err;
};

// A sequence as the kernels see it, brought within what the host said.
struct SeqView {
    int64_t row0;             // first query row
    int n, len;               // query rows, cached tokens
};

__device__ __forceinline__ SeqView seq_view(const AttendArgs &a, int64_t b, bool report) {
    SeqView v;
    int64_t r0 = a.q_start[b], r1 = a.q_start[b + 1];
    int64_t len = a.kv_len[b];
    bool bad = false;
    const int64_t cap = a.table_ld << a.g.page_shift;
    if (len < 0 || len > cap) {
        len = len < 0 ? 0 : cap;
        bad = true;
    }
    if (r0 < 0 || r1 < r0 || r1 > a.rows || r1 - r0 > a.max_q) {
        bad = true;
        r0 = r0 < 0 ? 0 : r0 > a.rows ? a.rows : r0;
        r1 = r1 < r0 ? r0 : r1 > a.rows ? a.rows : r1;
        if (r1 - r0 > a.max_q) r1 = r0 + a.max_q;
    }
    if (bad && report) set_error(a.err, ERR_RANGE);
    v.row0 = r0;
    v.n = static_cast<int>(r1 - r0);
    v.len = static_cast<int>(len);
    return v;
}

// Tokens that query rows i0 .. i1 (of n) see between them: [lo, hi), empty if hi <= lo.
__device__ __forceinline__ void visible(const AttendArgs &a, const SeqView &v, int i0, int i1, int &lo, int &hi) {
    lo = 0;
    hi = v.len;
    if (a.causal) {
        const int last = v.len - v.n + i1 + 1;
        hi = last < hi ? last : hi;
        if (a.window > 0) {
            const int64_t first = static_cast<int64_t>(v.len) - v.n + i0 - a.window + 1;
            lo = first > 0 ? static_cast<int>(first) : 0;
        }
    }
}

// Pieces of [lo, hi) in units of `unit` tokens (a power of two): tokens of a piece and how many there are.
__device__ __forceinline__ void pieces(const AttendArgs &a, int lo, int hi, int unit, int &size, int &count) {
    const int start = lo & ~(unit - 1);
    const int len = hi - start;
    if (hi <= lo) {
        size = unit;
        count = 0;
        return;
    }
    int per = (len + a.splits - 1) / a.splits;
    if (per < a.min_tokens) per = static_cast<int>(a.min_tokens);
    size = (per + unit - 1) & ~(unit - 1);
    count = (len + size - 1) / size;
}

// few query rows per kv head: warps of 16-token steps
cudaError_t launch_attend_rows(const AttendArgs &a, int tiles, int64_t row_chunks, cudaStream_t s);
// joins the pieces
cudaError_t launch_attend_join(const AttendArgs &a, int rows_per_chunk, int unit, cudaStream_t s);

}  // namespace qe
