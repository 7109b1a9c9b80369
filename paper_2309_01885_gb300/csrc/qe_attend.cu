// Attention over the 4-bit key/value cache: the entry points, how a call is cut up, and
// the joining of items that several workers share (kernels: qe_attend_rows.cuh for a few
// query rows to a kv head, qe_attend_tc.cu for many).
#include "qe_attend_rows.cuh"

namespace qe {
namespace {

// Joins the items that several workers share.  With a block for each item (by_item),
// or, where there are more items than workers, for each border between workers i and
// i + 1: that block takes the item which the border cuts, if it is its first border.
template <int N>
__global__ void __launch_bounds__(N) k_attend_join(const AttendArgs a, int unit, int by_item) {
    __shared__ int64_t sums[N + 1];
    __shared__ float4 meet_v[N];
    __shared__ float2 meet_s[N];
    if (a.first_pass) let_next_begin();
    int64_t share;
    scan_units<N>(a, unit, sums, share);
    const int64_t total = sums[N], per = worker_units(a, total);
    Place at;
    at.seq = -1;
    int64_t begin = 0, end = 0, item = 0, worker = 0;     // the item's units, and the worker that begins it
    bool cut = false;
    if (by_item) {
        const int of_seq = static_cast<int>(a.items / a.seqs);   // items of the longest sequence
        const int64_t seq = blockIdx.x / static_cast<unsigned>(of_seq);
        item = blockIdx.x - seq * of_seq;
        const SeqView v = seq_view(a, seq, false);
        const SeqWork w = seq_work(a, v, unit);
        if (item * w.steps < w.units) {
            at.seq = seq;
            at.v = v;
            at.w = w;
            const int of = static_cast<int>(share == 1 ? seq : div_small(seq, static_cast<int>(share)));
            at.base = sums[of];
            for (int64_t q = of * share; q < seq; ++q) at.base += seq_work(a, seq_view(a, q, false), unit).units;
            begin = at.base + item * w.steps;
            worker = per > 0x7fffffff ? begin / per : div_small(begin, static_cast<int>(per));
            end = begin + w.steps;
            cut = end > (worker + 1) * per;
        }
    } else {
        const int64_t border = (blockIdx.x + 1) * per;
        if (border < total) {
            locate<N>(a, unit, sums, share, border, at);
            item = div_small(border - at.base, at.w.steps);
            begin = at.base + item * at.w.steps;
            end = begin + at.w.steps;
            worker = blockIdx.x;
            cut = begin < border && begin >= border - per;
        }
    }
    wait_for_last();                                      // every block waits: the grid ends after the workers' grid
    if (!cut) return;
    const int count = 1 + static_cast<int>((per > 0x7fffffff ? (end - 1) / per : div_small(end - 1, static_cast<int>(per))) - worker);
    const int D = a.g.D, R = a.rows_cap;
    const int64_t size = static_cast<int64_t>(R) * (D + 2);
    const int chunk = static_cast<int>(div_small(item, a.g.kv_heads));
    const int kvh = static_cast<int>(item - static_cast<int64_t>(chunk) * a.g.kv_heads);
    const int first = chunk * R, all = at.v.n * a.per_kv;
    const int rows = all - first < R ? all - first : R;
    // this worker's piece begins the item (its second slot); the others continue it (their first ones)
    const float *base = a.part + 2 * worker * size;
    // threads beyond one for each four channels take every other (third, ...) piece and meet in shared memory
    const int quads = rows * (D / 4);
    int teams = quads <= N ? N / quads : 1;
    if (teams > count) teams = count;
    constexpr int AHEAD = 4;
    for (int i0 = 0; i0 < quads; i0 += N) {
        const int team = quads <= N ? static_cast<int>(threadIdx.x) / quads : 0;
        const int i = quads <= N ? static_cast<int>(threadIdx.x) - team * quads : i0 + static_cast<int>(threadIdx.x);
        const int row = i / (D / 4), d = 4 * (i % (D / 4));
        float big = kFloor, sum = 0.0f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        const bool on = i < quads && team < teams && d < a.g.dim;
        for (int s = team; on && s < count; s += AHEAD * teams) {
            float m[AHEAD], l[AHEAD];
            float4 u[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int q = s + k * teams;
                const float *p = base + (q == 0 ? 1 : 2 * q) * size;
                const bool here = q < count;
                m[k] = here ? p[R * D + row] : kFloor;
                l[k] = here ? p[R * (D + 1) + row] : 0.0f;
                u[k] = here ? *reinterpret_cast<const float4 *>(p + row * D + d) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            const float was = big;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) big = fmaxf(big, m[k]);
            const float keep = ex2(was - big);
            sum *= keep;
            v.x *= keep;
            v.y *= keep;
            v.z *= keep;
            v.w *= keep;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float f = ex2(m[k] - big);
                sum = fmaf(f, l[k], sum);
                v.x = fmaf(f, u[k].x, v.x);
                v.y = fmaf(f, u[k].y, v.y);
                v.z = fmaf(f, u[k].z, v.z);
                v.w = fmaf(f, u[k].w, v.w);
            }
        }
        if (teams > 1) {
            if (on && team > 0) {
                meet_v[threadIdx.x] = v;
                meet_s[threadIdx.x] = make_float2(big, sum);
            }
            __syncthreads();
            if (on && team == 0) {
                float top = big;
                for (int k = 1; k < teams; ++k) top = fmaxf(top, meet_s[k * quads + i].x);
                float f = ex2(big - top);
                sum *= f;
                v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                for (int k = 1; k < teams; ++k) {
                    const float2 q = meet_s[k * quads + i];
                    const float4 u = meet_v[k * quads + i];
                    f = ex2(q.x - top);
                    sum = fmaf(f, q.y, sum);
                    v = make_float4(fmaf(f, u.x, v.x), fmaf(f, u.y, v.y), fmaf(f, u.z, v.z), fmaf(f, u.w, v.w));
                }
                big = top;
            }
        }
        if (on && team == 0) {
            const unsigned pr = first + row, q = pr / static_cast<unsigned>(a.per_kv);
            finish(a, at.v, at.v.row0 + q, kvh * a.per_kv + static_cast<int>(pr - q * a.per_kv), d, v, big, sum);
        }
    }
}

cudaError_t launch_join(const AttendArgs &a, int unit, cudaStream_t s) {
    // few items among many workers have many pieces each: more threads share them
    const int threads = a.ctas > 4 * a.items ? 1024 : 256;
    const int by_item = a.items < a.ctas;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(by_item ? a.items : a.ctas - 1));
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute attr{};      // starts while the last workers run, and waits for them on the device
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return threads == 1024 ? cudaLaunchKernelEx(&cfg, k_attend_join<1024>, a, unit, by_item)
                           : cudaLaunchKernelEx(&cfg, k_attend_join<256>, a, unit, by_item);
}

}  // namespace

cudaError_t launch_attend_rows(const AttendArgs &a, int tiles, cudaStream_t s) {
    cudaError_t e = launch_rows_any<kDealtWarps, false>(a, tiles, s);
    if (e == cudaSuccess && a.ctas > 1) e = launch_join(a, kRowsUnit, s);
    return e;
}

}  // namespace qe

using namespace qe;

namespace {

// How a call is cut up.
struct AttendPlan {
    int tiles;                // 0: many rows, tiles of 128
    int rows_cap, ctas, min_units, splits;
    int warps;                // > 0: CTAs of so many warps take whole items
    int64_t items;            // at most
};

int sm_count() {
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

// (query row, head) pairs of a kv head up to which the few-rows kernel takes a call.  Measured (us on the GPU, few rows /
// tiles, caches out of L2, one row of so many heads on 8 kv heads): 2 x 30000 tokens, 64 channels 32 pairs 41 / 54, 33 pairs
// 56 / 54, 96 channels 50 / 63 and 67 / 63, 128 channels 59 / 70 and 79 / 70; 32 x 4096 tokens, 128 channels 101 / 143 and
// 137 / 143.
constexpr int kFewPairs = 32;

AttendPlan attend_plan(const CacheGeom &g, const qe_attention &at) {
    const int64_t seqs = at.seqs, max_q = at.max_q, max_kv = at.max_kv, window = at.causal ? at.window : 0;
    const int q_heads = at.q_heads;
    AttendPlan p;
    const int64_t pairs = max_q * (q_heads / g.kv_heads);
    const int64_t span = window > 0 && window + max_q < max_kv ? window + max_q : max_kv;   // most that a row sees
    p.splits = 1;
    p.warps = 0;
    if (pairs > kFewPairs) {
        p.tiles = 0;
        p.rows_cap = 256;
        p.items = seqs * ceil_div(pairs, 256) * g.kv_heads;
        p.ctas = 0;
        p.min_units = 4;
        // pieces of an item, each a CTA, while all of them fit one wave: 4 items of 53000 tokens 36 us.  Cutting for a
        // second wave as well does not pay where lengths differ: 160 items of 1000 .. 8000 tokens 150 us whole, 169 in
        // two pieces (of 8000 each: 295 and 267)
        const int64_t want = sm_count() / p.items, most = ceil_div(span, 128) / p.min_units;
        p.splits = static_cast<int>(want < most ? want : most);
        if (p.splits < 1) p.splits = 1;
        return p;
    }
    // registers: a tile of 8 rows costs 2 D / 32 accumulators and as much again for Q, so D > 64 takes two at most
    p.tiles = pairs <= 8 ? 1 : (pairs <= 16 || g.D > 64) ? 2 : 4;
    p.rows_cap = 8 * p.tiles;
    p.min_units = 8;
    const int64_t items = p.items = seqs * ceil_div(pairs, p.rows_cap) * g.kv_heads;
    // short contexts: a CTA for each item saves the dealing out and the joining.  Measured (us on 152 SMs, caches out of L2,
    // dealt out / CTAs of 8 warps / of 4; single tokens, 4 heads of 128 a kv head, lengths from half the span up): 32 items
    // of 2048 tokens 18 / 17 / 23, of 3000 18 / 23 / 32; 152 of 2048 26 / 18 / 24, of 4096 34 / 30 / 42; 160 of 1024
    // 25 / 19 / 16, of 1536 28 / 22 / 21; 512 of 1024 32 / 39 / 31, of 1536 37 / 49 / 41; 1216 of 512 42 / 57 / 40, of 1024
    // 60 / 85 / 62; 1280 of 512 43 / 61 / 45.  The limits are those of the most items of either form, and leave something to
    // fewer (160 of 1100: 25 for 17) and to smaller heads (64 channels, 1280 of 512: 32 for 24).
    p.warps = items <= sm_count() && span <= 2048 ? 8 : items <= 8 * sm_count() && span <= 1088 ? 4 : 0;
    if (p.warps > 0) {
        p.ctas = 1;
        return p;
    }
    const int64_t slots = static_cast<int64_t>(sm_count()) * rows_blocks(g.D / 32, p.tiles);
    const int64_t most = ceil_div(items * ceil_div(max_kv + kRowsUnit, kRowsUnit), p.min_units);
    p.ctas = static_cast<int>(most < slots ? most : slots);
    return p;
}

size_t attend_bytes(const AttendPlan &p, const CacheGeom &g) {
    if (p.tiles == 0) return p.splits == 1 ? 0 : static_cast<size_t>(p.items) * p.splits * p.rows_cap * (g.D + 2) * sizeof(float);
    if (p.ctas == 1) return 0;
    return static_cast<size_t>(2) * p.ctas * p.rows_cap * (g.D + 2) * sizeof(float);
}

int64_t smaller(int64_t a, int64_t b) { return a < b ? a : b; }

// The most that any batch needs which has no more sequences, query rows a sequence and tokens than this one.  (What one
// batch needs does not grow with it: 19 sequences may fill the GPU in whole items, which one alone has to be cut for.)
size_t attend_most_bytes(const CacheGeom &g, const qe_attention &at) {
    const int64_t pairs = at.max_q * (at.q_heads / g.kv_heads), row = static_cast<int64_t>(g.D + 2) * sizeof(float);
    int64_t most = 0;
    for (int tiles = 1; tiles <= (g.D <= 64 ? 4 : 2); tiles *= 2) {
        if (tiles > 1 && pairs <= 4 * tiles) break;       // no batch of these takes so many tiles
        const int cap = 8 * tiles;
        const int64_t end = tiles == (g.D <= 64 ? 4 : 2) ? kFewPairs : cap;
        const int64_t units = at.seqs * ceil_div(smaller(pairs, end), cap) * g.kv_heads * ceil_div(at.max_kv + kRowsUnit, kRowsUnit);
        const int64_t ctas = smaller(ceil_div(units, 8), static_cast<int64_t>(sm_count()) * rows_blocks(g.D / 32, tiles));
        if (ctas > 1 && 2 * ctas * cap * row > most) most = 2 * ctas * cap * row;
    }
    const int64_t pieces = ceil_div(at.max_kv, 128) / 4;  // of an item of tiles
    if (pairs > kFewPairs && pieces > 1 && sm_count() / g.kv_heads > 1) {
        const int64_t all = smaller(sm_count(), at.seqs * ceil_div(pairs, 256) * g.kv_heads * pieces) * 256 * row;
        if (all > most) most = all;
    }
    return static_cast<size_t>(most);
}

// Geometry of a cache that may have no memory yet (the workspace query takes it either way).
qe_status shape_geom(const qe_cache *cache, CacheGeom *g) {
    if (!cache) return QE_ERR_INVALID_ARG;
    qe_cache c = *cache;
    c.data = reinterpret_cast<void *>(static_cast<uintptr_t>(256));
    c.bytes = ~static_cast<size_t>(0);
    return cache_geom(&c, g);
}

qe_status check_shape(const CacheGeom &g, const qe_attention *at) {
    if (!at || at->seqs < 1 || at->rows < 0 || at->q_heads < 1 || at->max_q < 0 || at->max_kv < 0 || at->window < 0)
        return QE_ERR_INVALID_ARG;
    if (at->q_heads % g.kv_heads != 0 || (at->window > 0 && !at->causal)) return QE_ERR_INVALID_ARG;
    if (at->seqs > 65535 || at->rows > 0x7fffffff / at->q_heads || at->max_q > at->rows || at->max_kv > (1 << 30) ||
        at->window > (int64_t{1} << 31))
        return QE_ERR_INVALID_ARG;
    return QE_OK;
}

qe_status check_prefix(const qe_attention &at, int64_t prefix) {
    if (prefix < 0 || prefix > (1 << 30)) return QE_ERR_INVALID_ARG;
    return prefix > 0 && at.window > 0 ? QE_ERR_UNSUPPORTED : QE_OK;
}

cudaError_t launch_plan(AttendArgs a, const AttendPlan &p, cudaStream_t s) {
    a.rows_cap = p.rows_cap;
    a.ctas = p.ctas;
    a.items = p.items;
    a.splits = p.splits;
    a.min_units = p.min_units;
    return p.tiles == 0 ? launch_attend_tiles(a, s) : p.warps == 8   ? launch_attend_whole8(a, p.tiles, s)
           : p.warps == 4 ? launch_attend_whole4(a, p.tiles, s)
                          : launch_attend_rows(a, p.tiles, s);
}

// A prefix that sequences share is read once for all of them.  Attention over it, all rows of the batch as one sequence's
// without a mask, leaves unnormalised sums, maxima and totals in binary32; the pass over what is behind it joins them as it
// finishes its rows:  m = max(m1, m2),  o = (2^(m1 - m) o1 + 2^(m2 - m) o2) / (2^(m1 - m) l1 + 2^(m2 - m) l2).  The second pass
// does not need the first until it finishes: it is launched to begin while the first one's last blocks run.  Measured (us, 32
// heads of 128 on 8, one row each): 64 sequences behind 8192 tokens with up to 1000 of their own 64, with up to 100 48 (81 and 67
// one after the other); 200 behind 16000 with 500 .. 6000 304 (310).

// The prefix's pass, all rows of the batch as one sequence's, and the one over what is behind it.
qe_attention front_of(const qe_attention &at, int64_t prefix) {
    qe_attention f = at;
    f.seqs = 1;
    f.max_q = at.rows;
    f.max_kv = prefix;
    f.causal = 0;
    f.window = 0;
    return f;
}

qe_attention back_of(const qe_attention &at, int64_t prefix) {
    qe_attention b = at;
    b.max_kv = at.max_kv > prefix ? at.max_kv - prefix : 0;
    return b;
}

size_t first_bytes(const CacheGeom &g, const qe_attention &at) {
    return static_cast<size_t>(round_up(at.rows * at.q_heads * (g.D + 2) * static_cast<int64_t>(sizeof(float)), 256));
}

// Attention, with `shared` tokens in prefix_pages before each sequence's own where these are given.
qe_status attend(const qe_cache *cache, const qe_attention *at, const int32_t *prefix_pages, int64_t shared, const void *Q, int64_t q_row,
                 int64_t q_head, void *out, int64_t o_row, int64_t o_head, qe_dtype dtype, float *lse, void *workspace,
                 size_t workspace_bytes, qe_stream_t stream) {
    AttendArgs a{};
    qe_status st = cache_geom(cache, &a.g);
    if (st != QE_OK) return st;
    if ((st = check_shape(a.g, at)) != QE_OK) return st;
    if (dtype != QE_BF16 && dtype != QE_F16) return dtype == QE_F32 ? QE_ERR_UNSUPPORTED : QE_ERR_INVALID_ARG;
    if (at->rows == 0 || at->max_q == 0) return QE_OK;
    if (!at->q_start || !at->kv_len || !at->page_table || at->table_ld < 1 || !Q || !out) return QE_ERR_INVALID_ARG;
    if (at->table_ld > (int64_t{1} << 30) >> a.g.page_shift) return QE_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(out)) & 1u) != 0 ||
        ((reinterpret_cast<uintptr_t>(at->q_start) | reinterpret_cast<uintptr_t>(at->kv_len) |
          reinterpret_cast<uintptr_t>(at->page_table) | reinterpret_cast<uintptr_t>(lse)) & 3u) != 0 ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
        return QE_ERR_INVALID_ARG;
    if (!(at->scale >= 0.0f) || at->scale > 1e30f) return QE_ERR_INVALID_ARG;
    a.q_start = at->q_start;
    a.kv_len = at->kv_len;
    a.table = at->page_table;
    a.table_ld = at->table_ld;
    a.rows = at->rows;
    a.seqs = at->seqs;
    a.max_q = at->max_q;
    a.q_heads = at->q_heads;
    a.per_kv = at->q_heads / a.g.kv_heads;
    a.causal = at->causal != 0;
    a.window = at->window;
    a.scale2 = (at->scale > 0.0f ? at->scale : 1.0f / sqrtf(static_cast<float>(a.g.dim))) * 1.44269504088896341f;
    a.Q = Q;
    a.out = out;
    a.q_row = q_row;
    a.q_head = q_head;
    a.o_row = o_row;
    a.o_head = o_head;
    a.half = dtype == QE_F16;
    a.q_vec = (reinterpret_cast<uintptr_t>(Q) & 15u) == 0 && q_row % 8 == 0 && q_head % 8 == 0;
    a.o_vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && o_row % 8 == 0 && o_head % 8 == 0;
    a.lse = lse;
    a.err = device_error_word();
    if (!a.err) return QE_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const int64_t prefix = prefix_pages ? shared : 0;
    const AttendPlan p = attend_plan(a.g, back_of(*at, prefix));
    AttendPlan p1{};
    if (prefix > 0) p1 = attend_plan(a.g, front_of(*at, prefix));
    // the workers' unfinished items, of either pass, lie behind what the first pass leaves
    const size_t kept = prefix > 0 ? first_bytes(a.g, *at) : 0;
    size_t need = attend_bytes(p, a.g);
    if (prefix > 0 && attend_bytes(p1, a.g) > need) need = attend_bytes(p1, a.g);
    need += kept;
    void *own = nullptr;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (need > 0) {
        if (workspace) {
            if (workspace_bytes < need) return QE_ERR_OOM;
        } else {
            if (cudaMallocAsync(&own, need, s) != cudaSuccess) {
                cudaGetLastError();
                return QE_ERR_OOM;
            }
            ws = static_cast<uint8_t *>(own);
        }
        a.part = reinterpret_cast<float *>(ws + kept);
    }
    cudaError_t e = cudaSuccess;
    if (prefix > 0) {
        a.prefix = static_cast<int>(prefix);
        a.first = reinterpret_cast<float *>(ws);
        AttendArgs f = a;
        f.first_pass = 1;
        f.batch_seqs = at->seqs;
        f.seqs = 1;
        f.max_q = at->rows;
        f.causal = 0;
        f.table = prefix_pages;
        f.table_ld = ceil_div(prefix, int64_t{1} << a.g.page_shift);
        e = launch_plan(f, p1, s);
    }
    if (e == cudaSuccess) e = launch_plan(a, p, s);
    if (own) cudaFreeAsync(own, s);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return QE_ERR_CUDA;
    }
    return QE_OK;
}

}  // namespace

extern "C" {

qe_status qe_cache_attention_workspace(const qe_cache *cache, const qe_attention *at, size_t *bytes) {
    CacheGeom g;
    if (!bytes) return QE_ERR_INVALID_ARG;
    qe_status st = shape_geom(cache, &g);
    if (st != QE_OK) return st;
    if ((st = check_shape(g, at)) != QE_OK) return st;
    *bytes = attend_most_bytes(g, *at);
    return QE_OK;
}

qe_status qe_cache_attention(const qe_cache *cache, const qe_attention *at, const void *Q, int64_t q_row, int64_t q_head,
                             void *out, int64_t o_row, int64_t o_head, qe_dtype dtype, float *lse, void *workspace,
                             size_t workspace_bytes, qe_stream_t stream) {
    return attend(cache, at, nullptr, 0, Q, q_row, q_head, out, o_row, o_head, dtype, lse, workspace, workspace_bytes, stream);
}

qe_status qe_cache_attention_shared_workspace(const qe_cache *cache, const qe_attention *at, int64_t prefix, size_t *bytes) {
    CacheGeom g;
    if (!bytes) return QE_ERR_INVALID_ARG;
    qe_status st = shape_geom(cache, &g);
    if (st != QE_OK) return st;
    if ((st = check_shape(g, at)) != QE_OK) return st;
    if ((st = check_prefix(*at, prefix)) != QE_OK) return st;
    const size_t back = attend_most_bytes(g, *at), front = attend_most_bytes(g, front_of(*at, prefix));   // (a shorter prefix leaves more)
    *bytes = (back > front ? back : front) + first_bytes(g, *at);
    return QE_OK;
}

qe_status qe_cache_attention_shared(const qe_cache *cache, const qe_attention *at, const int32_t *prefix_pages, int64_t prefix,
                                    const void *Q, int64_t q_row, int64_t q_head, void *out, int64_t o_row, int64_t o_head,
                                    qe_dtype dtype, float *lse, void *workspace, size_t workspace_bytes, qe_stream_t stream) {
    if (!at) return QE_ERR_INVALID_ARG;
    const qe_status st = check_prefix(*at, prefix);
    if (st != QE_OK) return st;
    if (prefix > 0 && (!prefix_pages || (reinterpret_cast<uintptr_t>(prefix_pages) & 3u) != 0)) return QE_ERR_INVALID_ARG;
    return attend(cache, at, prefix > 0 ? prefix_pages : nullptr, prefix, Q, q_row, q_head, out, o_row, o_head, dtype, lse, workspace,
                  workspace_bytes, stream);
}

}  // extern "C"
