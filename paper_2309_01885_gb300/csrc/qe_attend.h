// Arguments and launchers of attention over the 4-bit key/value cache.
#pragma once

#include <atomic>

#include "qe_cache.cuh"

namespace qe {

struct AttendArgs {
    CacheGeom g;
    const int32_t *q_start, *kv_len, *table;
    int64_t table_ld;
    int64_t rows;             // query rows in all; rows x q_heads < 2^31
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
    int q_vec, o_vec;         // 16-byte loads of Q, stores of out are aligned
    float *lse;               // [rows][q_heads], natural log, or NULL
    int rows_cap;             // (query row, head) pairs that an item of work holds
    int ctas;                 // workers among which the units are dealt out
    int64_t items;            // how many items there may be
    int min_units;            // a worker (or a piece) takes at least this many
    int splits;               // tiles of 128 rows: pieces of an item's tokens
    float *part;              // unfinished items: [2 ctas][rows_cap x D sums, rows_cap maxima, rows_cap totals]
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

// x / y for 0 <= x, 0 < y < 2^31: in 32 bits where x fits, which takes a tenth of the time.
__device__ __forceinline__ int64_t div_small(int64_t x, int y) {
    if ((x >> 32) == 0) return static_cast<uint32_t>(x) / static_cast<uint32_t>(y);
    return x / y;
}

// The work as a line of units.  An item is one kv head of one sequence with up to
// rows_cap of the (query row, head of the group) pairs that read it; its units are
// the `unit`-token steps over the tokens that the sequence's rows see.  Items of a
// sequence have the same number of units (one, an empty one, where rows see nothing)
// and lie next to each other, kv heads fastest; worker i takes the units
// [i per, (i + 1) per), whatever lengths the batch has.
struct SeqWork {
    int64_t units;            // of all its items
    int steps;                // of one item
    int lo, hi;               // tokens its rows see between them
};

__device__ __forceinline__ SeqWork seq_work(const AttendArgs &a, const SeqView &v, int unit) {
    SeqWork w;
    w.units = 0;
    w.steps = 1;
    w.lo = w.hi = 0;
    if (v.n == 0) return w;
    visible(a, v, 0, v.n - 1, w.lo, w.hi);
    const int start = w.lo & ~(unit - 1);
    if (w.hi > w.lo) w.steps = (w.hi - start + unit - 1) / unit;
    const int chunks = (v.n * a.per_kv + a.rows_cap - 1) / a.rows_cap;     // rows x heads < 2^31
    w.units = static_cast<int64_t>(chunks) * a.g.kv_heads * w.steps;
    return w;
}

// Sums of the units before thread i's share of the sequences, for N threads; total in out[N].
template <int N>
__device__ __forceinline__ void scan_units(const AttendArgs &a, int unit, int64_t *out, int64_t &share) {
    share = (a.seqs + N - 1) / N;
    int64_t mine = 0;
    for (int64_t b = threadIdx.x * share; b < (threadIdx.x + 1) * share && b < a.seqs; ++b)
        mine += seq_work(a, seq_view(a, b, blockIdx.x == 0), unit).units;
    int64_t sum = mine;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
    }
    if (lane == 31) out[1 + (threadIdx.x >> 5)] = sum;    // warp totals, for the moment
    __syncthreads();
    int64_t before = 0;
    for (int w = 0; w < static_cast<int>(threadIdx.x >> 5); ++w) before += out[1 + w];
    __syncthreads();
    out[1 + threadIdx.x] = before + sum;
    if (threadIdx.x == 0) out[0] = 0;
    __syncthreads();
}

// A place on the line: which sequence, and the units before it.
struct Place {
    int64_t seq, base;
    SeqView v;
    SeqWork w;
};

// The sequence that unit `pos` (below the total) belongs to; `p` may hold an earlier place to go on from (seq >= 0).
template <int N>
__device__ __forceinline__ void locate(const AttendArgs &a, int unit, const int64_t *sums, int64_t share, int64_t pos, Place &p) {
    if (p.seq >= 0 && pos < p.base + p.w.units) return;
    int lo = 0, hi = N;                                   // sums[lo] <= pos < sums[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= pos) lo = mid;
        else hi = mid;
    }
    p.base = sums[lo];
    for (p.seq = lo * share;; ++p.seq) {
        p.v = seq_view(a, p.seq, false);
        p.w = seq_work(a, p.v, unit);
        if (pos < p.base + p.w.units || p.seq + 1 >= a.seqs) break;
        p.base += p.w.units;
    }
}

__device__ __forceinline__ int64_t worker_units(const AttendArgs &a, int64_t total) {
    const int64_t per = div_small(total + a.ctas - 1, a.ctas);
    return per < a.min_units ? a.min_units : per;
}

// Raises a kernel's limit of dynamic shared memory on the current device, once a device (the call takes longer than the
// question whether it has been made); `raised`, a bit a device, is the kernel's own.  A refusal is not remembered.
inline cudaError_t raise_smem(const void *kernel, int bytes, std::atomic<uint64_t> &raised) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (raised.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// few query rows per kv head: `tiles` x 8 pairs an item; then the items that workers share are joined
cudaError_t launch_attend_rows(const AttendArgs &a, int tiles, cudaStream_t s);
// the same with a CTA (of 8 or 4 warps) for each item
cudaError_t launch_attend_whole8(const AttendArgs &a, int tiles, cudaStream_t s);
cudaError_t launch_attend_whole4(const AttendArgs &a, int tiles, cudaStream_t s);
constexpr int kRowsUnit = 32;

// many query rows per kv head: tiles of 128 rows on the tensor cores
cudaError_t launch_attend_tiles(const AttendArgs &a, cudaStream_t s);

}  // namespace qe
