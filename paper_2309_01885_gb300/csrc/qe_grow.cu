// Pages, slots and positions of a batch's new tokens, from their lengths alone.
//
// With l_b the tokens sequence b keeps and n_b those it takes, everything is a place in
// one of three running sums over the sequences: tokens (n_b), pages taken (ceil((l_b +
// n_b) / P) - ceil(l_b / P)) and pages given back.  One block forms the sums, 1024
// threads with neighbouring sequences each, checks the call, moves the pages that come
// back and writes the lengths.  Then a thread per token finds its sequence by bisection
// over q_start; a token that begins a page also enters the page in the table, so every
// new page is entered once.  Pages that come back go behind those that wait, so no
// thread reads a place of the ring that another writes.  Up to kAlone tokens the same
// block does that too (one launch); more are spread over the GPU by a second one that is
// started early and waits on the device.
//
// Bound by latency: a few kilobytes are read and written, through a chain of dependent
// steps (read lengths, scan, bisection over q_start: 6 reads for 64 sequences, 11 for 1500, read the
// ring, write).  64 sequences of a token each 8 us, 1500 of 100
// (150000 tokens) 14 us.
#include "qe_cache.cuh"
#include "qe_internal.h"

namespace qe {
namespace {

constexpr int kThreads = 1024;
// Measured (us, one block / spread): 64 tokens 8 / 10, 1024 8 / 10, 2048 12 / 14, 4096 18 / 16 (of 4096 sequences; of 32 10 / 10),
// 8192 16 / 10, 150000 188 / 14.
constexpr int kAlone = 2048;

struct GrowArgs {
    int64_t pages, cells;     // of the ring; tokens that fit a row of the table
    int page_shift;
    int seqs, max_tokens, prefix;
    int64_t table_ld;
    const int32_t *new_tokens, *kv_len, *state;
    const uint8_t *ends;
    int32_t *kv_len_out, *table, *ring, *state_out, *q_start, *positions;
    int64_t *slots;
    int32_t *keep;            // workspace: l_b
    int32_t *taken;           // workspace: pages that earlier sequences take; behind them ring's first and whether all is well
    unsigned *err;
};

struct Sums {
    int64_t tokens, taken, back;
};

__device__ __forceinline__ int pages_of(const GrowArgs &a, int64_t tokens) {
    return static_cast<int>((tokens + (int64_t{1} << a.page_shift) - 1) >> a.page_shift);
}

// A sequence's lengths and pages; false where they do not fit.
__device__ __forceinline__ bool sequence(const GrowArgs &a, int b, int &n, int &keep, int &taken, int &back) {
    n = a.new_tokens[b];
    const int len = a.kv_len[b];
    const bool over = a.ends && a.ends[b] != 0;
    keep = over ? a.prefix : len;
    taken = back = 0;
    if (n < 0 || len < 0 || len > a.cells || static_cast<int64_t>(keep) + n > a.cells) return false;
    taken = pages_of(a, static_cast<int64_t>(keep) + n) - pages_of(a, keep);
    if (over) back = max(pages_of(a, len) - (a.prefix >> a.page_shift), 0);
    return true;
}

__device__ __forceinline__ int64_t wrapped(int64_t at, int64_t pages) { return at >= pages ? at - pages : at; }

// The token's sequence, position and slot, and its page where it begins one.
__device__ __forceinline__ void token(const GrowArgs &a, int i, int total, int64_t first) {
    int64_t slot = -1;
    int at = 0;
    if (i < total) {
        int lo = 0, hi = a.seqs;                          // q_start[lo] <= i < q_start[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.q_start[mid] <= i) lo = mid;
            else hi = mid;
        }
        const int keep = a.keep[lo];
        at = keep + (i - a.q_start[lo]);
        const int k = at >> a.page_shift, fresh = k - pages_of(a, keep);
        int32_t *cell = a.table + lo * a.table_ld + k;
        int page;
        if (fresh >= 0) {
            page = a.ring[wrapped(first + a.taken[lo] + fresh, a.pages)];
            // (the first of the page: of the sequence's tokens or of the page itself)
            if ((at & ((1 << a.page_shift) - 1)) == 0) *cell = page;
        } else {
            page = *cell;
        }
        slot = (static_cast<int64_t>(page) << a.page_shift) + (at & ((1 << a.page_shift) - 1));
        if (page < 0) slot = -1;
    }
    a.slots[i] = slot;
    if (a.positions) a.positions[i] = at;
}

__device__ __forceinline__ Sums warp_scan(Sums v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, v.tokens, o), y = __shfl_up_sync(0xffffffffu, v.taken, o),
                      z = __shfl_up_sync(0xffffffffu, v.back, o);
        if (lane >= o) {
            v.tokens += x;
            v.taken += y;
            v.back += z;
        }
    }
    return v;
}

// alone: this block does the tokens too.
__global__ void __launch_bounds__(kThreads) k_grow_sums(const GrowArgs a, int alone) {
    __shared__ Sums of_warp[32];
    __shared__ Sums all;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int share = (a.seqs + kThreads - 1) / kThreads;
    const int begin = min(static_cast<int>(threadIdx.x) * share, a.seqs), end = min(begin + share, a.seqs);
    bool fits = true;
    Sums mine{0, 0, 0};
    for (int b = begin; b < end; ++b) {
        int n, keep, taken, back;
        fits = sequence(a, b, n, keep, taken, back) && fits;
        mine.tokens += n;
        mine.taken += taken;
        mine.back += back;
    }
    const int64_t first = a.state[0], count = a.state[1];
    const Sums upto = warp_scan(mine);
    if (lane == 31) of_warp[warp] = upto;
    fits = __syncthreads_and(fits);                       // (every thread has read the state by now)
    if (warp == 0) {
        const Sums w = warp_scan(of_warp[lane]);
        if (lane == 31) all = w;
        Sums before = w;
        before.tokens -= of_warp[lane].tokens;
        before.taken -= of_warp[lane].taken;
        before.back -= of_warp[lane].back;
        __syncwarp();
        of_warp[lane] = before;
    }
    __syncthreads();
    if (fits)
        fits = all.tokens <= a.max_tokens && first >= 0 && first < a.pages && count >= 0 && all.taken <= count &&
               count + all.back <= a.pages;
    Sums at{of_warp[warp].tokens + upto.tokens - mine.tokens, of_warp[warp].taken + upto.taken - mine.taken,
            of_warp[warp].back + upto.back - mine.back};
    for (int k = 0; k < share; ++k) {                     // (the warp's lanes go along together)
        const int b = begin + k;
        const bool on = b < end;
        int n = 0, keep = 0, taken = 0, back = 0;
        if (on && fits) {
            sequence(a, b, n, keep, taken, back);
            a.keep[b] = keep;
            a.taken[b] = static_cast<int>(at.taken);
            a.q_start[b] = static_cast<int>(at.tokens);
        } else if (on) {
            a.q_start[b] = 0;
            a.kv_len_out[b] = a.kv_len[b];
        }
        // pages that come back: the whole warp moves one sequence's after the other
        const int64_t to = wrapped(wrapped(first + count, a.pages) + at.back, a.pages);
        for (unsigned some = __ballot_sync(0xffffffffu, back > 0); some != 0u; some &= some - 1u) {
            const int src = __ffs(static_cast<int>(some)) - 1;
            const int of = __shfl_sync(0xffffffffu, b, src), m = __shfl_sync(0xffffffffu, back, src);
            const int64_t put = __shfl_sync(0xffffffffu, to, src);
            const int32_t *from = a.table + of * a.table_ld + (a.prefix >> a.page_shift);
            for (int i = lane; i < m; i += 32) a.ring[wrapped(put + i, a.pages)] = from[i];
        }
        if (on && fits) a.kv_len_out[b] = keep + n;
        at.tokens += n;
        at.taken += taken;
        at.back += back;
    }
    if (threadIdx.x == 0) {
        a.q_start[a.seqs] = fits ? static_cast<int>(all.tokens) : 0;
        a.taken[a.seqs] = static_cast<int>(first);
        a.state_out[0] = static_cast<int>(fits ? wrapped(first + all.taken, a.pages) : first);
        a.state_out[1] = static_cast<int>(fits ? count - all.taken + all.back : count);
        if (!fits) set_error(a.err, ERR_RANGE);
    }
    if (!alone) return;
    __syncthreads();
    const int total = fits ? static_cast<int>(all.tokens) : 0;
    for (int i = threadIdx.x; i < a.max_tokens; i += kThreads) token(a, i, total, first);
}

__global__ void __launch_bounds__(256) k_grow_tokens(const GrowArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < a.max_tokens) token(a, i, a.q_start[a.seqs], a.taken[a.seqs]);
}

size_t grow_bytes(int64_t seqs) { return static_cast<size_t>(round_up(4 * seqs, 256) + round_up(4 * (seqs + 1), 256)); }

bool misaligned(const void *p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

}  // namespace
}  // namespace qe

using namespace qe;

extern "C" {

qe_status qe_cache_grow_workspace(int64_t seqs, size_t *bytes) {
    if (!bytes || seqs < 1 || seqs > 65535) return QE_ERR_INVALID_ARG;
    *bytes = grow_bytes(seqs);
    return QE_OK;
}

qe_status qe_cache_grow(const qe_cache *cache, const qe_growth *gr, void *workspace, size_t workspace_bytes, qe_stream_t stream) {
    CacheGeom g;
    const qe_status st = cache_geom(cache, &g);
    if (st != QE_OK) return st;
    if (!gr || gr->seqs < 1 || gr->seqs > 65535 || gr->max_tokens < 0 || gr->max_tokens > (1 << 30) || gr->prefix < 0 ||
        gr->prefix > (1 << 30) || gr->prefix % cache->page_size != 0 || gr->table_ld < 1 ||
        gr->table_ld > (int64_t{1} << 30) >> g.page_shift)
        return QE_ERR_INVALID_ARG;
    if (!gr->new_tokens || !gr->kv_len || !gr->kv_len_out || !gr->page_table || !gr->ring || !gr->state || !gr->state_out ||
        !gr->q_start || (!gr->slots && gr->max_tokens > 0))
        return QE_ERR_INVALID_ARG;
    if (misaligned(gr->new_tokens, 3) || misaligned(gr->kv_len, 3) || misaligned(gr->kv_len_out, 3) || misaligned(gr->page_table, 3) ||
        misaligned(gr->ring, 3) || misaligned(gr->state, 3) || misaligned(gr->state_out, 3) || misaligned(gr->q_start, 3) ||
        misaligned(gr->positions, 3) || misaligned(gr->slots, 7) || misaligned(workspace, 255))
        return QE_ERR_INVALID_ARG;
    if (gr->prefix > gr->table_ld << g.page_shift) return QE_ERR_INVALID_ARG;
    const size_t need = grow_bytes(gr->seqs);
    if (workspace && workspace_bytes < need) return QE_ERR_OOM;
    GrowArgs a{};
    a.pages = g.pages;
    a.cells = gr->table_ld << g.page_shift;
    a.page_shift = g.page_shift;
    a.seqs = static_cast<int>(gr->seqs);
    a.max_tokens = static_cast<int>(gr->max_tokens);
    a.prefix = static_cast<int>(gr->prefix);
    a.table_ld = gr->table_ld;
    a.new_tokens = gr->new_tokens;
    a.kv_len = gr->kv_len;
    a.state = gr->state;
    a.ends = gr->ends;
    a.kv_len_out = gr->kv_len_out;
    a.table = gr->page_table;
    a.ring = gr->ring;
    a.state_out = gr->state_out;
    a.q_start = gr->q_start;
    a.positions = gr->positions;
    a.slots = gr->slots;
    a.err = device_error_word();
    if (!a.err) return QE_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    void *own = nullptr;
    if (!workspace && cudaMallocAsync(&own, need, s) != cudaSuccess) {
        cudaGetLastError();
        return QE_ERR_OOM;
    }
    a.keep = static_cast<int32_t *>(workspace ? workspace : own);
    a.taken = a.keep + round_up(4 * gr->seqs, 256) / 4;
    const int alone = gr->max_tokens <= kAlone;
    k_grow_sums<<<1, kThreads, 0, s>>>(a, alone);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess && !alone) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(gr->max_tokens, 256)));
        cfg.blockDim = dim3(256);
        cfg.stream = s;
        cudaLaunchAttribute attr{};      // starts while the sums are formed, and waits for them on the device
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, k_grow_tokens, a);
    }
    if (own) cudaFreeAsync(own, s);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return QE_ERR_CUDA;
    }
    return QE_OK;
}

}  // extern "C"
