"""The 4-bit key/value cache on the GPU: what it stores, what it gives back, and attention over it,
against plain forms of the definitions (binary32 where the definition is binary32, else binary64)."""
import math

import numpy as np
import pytest
import torch

from paper_2309_01885_gb300 import build, qe

pytestmark = pytest.mark.gpu

SIZES = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}   # ulp of a value in [1, 2)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def stored(x, group):
    """s (c - z) of x (tokens x heads x dim), each step in IEEE binary32 as the definition says."""
    x = x.float().cpu().numpy()
    n, h, dim = x.shape
    D = 64 if dim <= 64 else 96 if dim <= 96 else 128
    y = np.zeros((n, h, D), np.float32)
    y[..., :dim] = x
    y = y.reshape(n, h, D // group, group)
    lo, hi = np.minimum(y.min(-1), np.float32(0)), np.maximum(y.max(-1), np.float32(0))
    r = torch.from_numpy((hi - lo) / np.float32(15)).to(torch.bfloat16).float().numpy()
    s = np.maximum(r, np.float32(2.0 ** -126))[..., None]
    z = np.rint(-lo[..., None] / s)
    c = np.clip(np.rint(y / s) + z, 0, 15).astype(np.float32)
    return torch.from_numpy((s * (c - z)).reshape(n, h, D)[..., :dim].copy())


def filled(pages, page, heads, dim, group, seed=0, garbage=True):
    """A cache whose unwritten bytes are all ones: NaN scales and zero points wherever nothing was written."""
    c = qe.KVCache(pages, page, heads, dim, group)
    c.data.fill_(0xFF if garbage else 0)
    return c


@pytest.mark.parametrize("dim,group,page,heads,dtype", [
    (128, 32, 64, 3, torch.bfloat16), (128, 64, 16, 1, torch.float16), (128, 128, 128, 2, torch.float32),
    (64, 32, 32, 5, torch.float16), (64, 64, 256, 8, torch.bfloat16), (96, 32, 16, 3, torch.float32),
    (80, 32, 64, 4, torch.bfloat16), (72, 32, 32, 2, torch.float32), (8, 64, 16, 3, torch.float16),
    (120, 128, 64, 1, torch.bfloat16)])
@pytest.mark.parametrize("tokens", [1, 7, 131])
def test_read_gives_what_the_definition_stores(dim, group, page, heads, dtype, tokens):
    g = gen(tokens * 7 + dim)
    pages = tokens // page + 3
    c = filled(pages, page, heads, dim, group)
    fused = torch.randn(tokens, 2 * heads + 1, dim, generator=g, device="cuda") * 3 + 1
    fused[: tokens // 3] *= 1e-3
    fused = fused.to(dtype)
    k, v = fused[:, 1:1 + heads], fused[:, 1 + heads:]
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    before = c.data.clone()
    qe.qe_cache_append(c, k, v, slots)
    for out in (torch.float32, torch.bfloat16, torch.float16):
        kr, vr = qe.qe_cache_read(c, slots, out)
        assert torch.equal(kr.cpu(), stored(k, group).to(out)) and torch.equal(vr.cpu(), stored(v, group).to(out))
    assert qe.qe_sync_status() == qe.QE_OK
    # appending again what was stored elsewhere leaves every other byte as it was
    other = filled(pages, page, heads, dim, group)
    qe.qe_cache_append(other, k, v, slots)
    assert torch.equal(other.data, c.data)
    D = 64 if dim <= 64 else 96 if dim <= 96 else 128
    assert (c.data != before).sum().item() <= tokens * heads * (D + 8 * (D // group))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_groups_at_the_ends_of_the_range(dtype):
    """All zeros, one-sided groups, one outlier, exact midpoints, the smallest and the largest magnitudes."""
    big = 60000.0 if dtype == torch.float16 else 2.0 ** 126
    rows = [torch.zeros(64), torch.full((64,), 2.5), torch.full((64,), -1.25), torch.linspace(-1, 1, 64),
            torch.linspace(0, 15, 31).repeat(3)[:64], torch.cat([torch.tensor([1000.0]), torch.full((63,), 0.01)]),
            torch.linspace(-big, big, 64), torch.linspace(-1, 1, 64) * 2.0 ** -14,
            torch.linspace(-1, 1, 64) * (2.0 ** -149 * 100 if dtype == torch.float32 else 2.0 ** -24)]
    x = torch.stack(rows)[:, None].to(dtype).cuda()
    c = filled(2, 16, 1, 64, 32)
    slots = torch.arange(len(rows), device="cuda") + 5
    qe.qe_cache_append(c, x, -x, slots)
    k, v = qe.qe_cache_read(c, slots, torch.float32)
    assert qe.qe_sync_status() == qe.QE_OK
    assert torch.equal(k.cpu(), stored(x, 32)) and torch.equal(v.cpu(), stored(-x, 32))
    assert k.isfinite().all()
    # every value is within half a step (and the rounding of the scale) of what was written
    lo, hi = x.float().unflatten(-1, (2, 32)).amin(-1).clamp(max=0), x.float().unflatten(-1, (2, 32)).amax(-1).clamp(min=0)
    step = (hi.double() - lo.double()) / 15
    err = (k.double() - x.double()).abs().unflatten(-1, (2, 32))
    assert (err <= step[..., None] * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -126).all()


def test_strides_alignment_and_order_do_not_matter():
    n, h, dim = 37, 3, 80
    g = gen(3)
    x = torch.randn(n, h, dim, generator=g, device="cuda").to(torch.bfloat16)
    y = torch.randn(n, h, dim, generator=g, device="cuda").to(torch.bfloat16)
    slots = torch.randperm(128, generator=g, device="cuda")[:n]
    want = filled(8, 16, h, dim, 32)
    qe.qe_cache_append(want, x, y, slots)
    odd = torch.zeros(n * h * (dim + 3) + 1, dtype=torch.bfloat16, device="cuda")[1:].view(n, h, dim + 3)[..., :dim]
    odd.copy_(x)
    turned = y.permute(1, 0, 2).contiguous().permute(1, 0, 2)       # head-major memory
    got = filled(8, 16, h, dim, 32)
    order = torch.randperm(n, generator=g, device="cuda")
    qe.qe_cache_append(got, odd, turned, slots)
    assert torch.equal(got.data, want.data)
    got = filled(8, 16, h, dim, 32)
    qe.qe_cache_append(got, x[order], y[order], slots[order])
    assert torch.equal(got.data, want.data)
    # outputs into strided, unaligned tensors, nothing beside them touched
    full = torch.full((n, h, dim + 5), 7.0, dtype=torch.float16, device="cuda")
    turned = torch.full((h, n, dim), 7.0, dtype=torch.float16, device="cuda").permute(1, 0, 2)
    k, v = qe.qe_cache_read(want, slots, torch.float16, k=full[..., 3:3 + dim], v=turned)
    kr, vr = qe.qe_cache_read(want, slots, torch.float16)
    assert torch.equal(k, kr) and torch.equal(v, vr) and (full[..., :3] == 7).all() and (full[..., 3 + dim:] == 7).all()


def test_skipped_and_refused_slots():
    c = filled(2, 16, 2, 64, 64)
    x = torch.randn(6, 2, 64, generator=gen(4), device="cuda")
    before = c.data.clone()
    qe.qe_cache_append(c, x, x, torch.tensor([-1, -5, -1, -1, -1, -(1 << 40)], device="cuda"))
    assert qe.qe_sync_status() == qe.QE_OK and torch.equal(c.data, before)
    slots = torch.tensor([0, 32, 31, 1 << 33, -1, 7], device="cuda")
    qe.qe_cache_append(c, x, x, slots)
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG and qe.qe_sync_status() == qe.QE_OK
    k, v = qe.qe_cache_read(c, slots, torch.float32)
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG
    want = stored(x, 64)
    want[[1, 3, 4]] = 0
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), want)
    qe.qe_cache_append(c, x[:0], x[:0], slots[:0])
    assert qe.qe_cache_read(c, slots[:0])[0].shape == (0, 2, 64) and qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 2.0 ** 127])
def test_non_finite_values_are_marked_and_reported(value):
    c = filled(2, 16, 2, 128, 32)
    x = torch.randn(4, 2, 128, generator=gen(5), device="cuda")
    y = x.clone()
    y[2, 1, 77] = value
    slots = torch.arange(4, device="cuda")
    for k, v in ((x, y), (y, x)):
        qe.qe_cache_append(c, k, v, slots)
        assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
        kr, vr = qe.qe_cache_read(c, slots, torch.bfloat16)
        for got in (kr, vr):
            assert got[2, 1].isnan().all()
            good = torch.ones(4, 2, dtype=torch.bool)
            good[2, 1] = False
            assert torch.equal(got.cpu()[good], stored(x, 32).to(torch.bfloat16)[good])
    qe.qe_cache_append(c, x, x, slots)          # written over, the slot is good again
    assert qe.qe_sync_status() == qe.QE_OK and torch.equal(qe.qe_cache_read(c, slots, torch.float32)[0].cpu(), stored(x, 32))


# ---- attention ---------------------------------------------------------------------------------

class Batch:
    """A ragged batch over a paged cache: pages in random order, garbage wherever nothing was written."""

    def __init__(self, q_len, kv_len, heads, kv_heads, dim, group, page, dtype, seed=0, spread=1.0):
        g = gen(1000 + seed)
        self.q_len, self.kv_len, self.heads, self.dim = q_len, kv_len, heads, dim
        need = [-(-n // page) for n in kv_len]
        pages = sum(need) + 3
        self.cache = filled(pages, page, kv_heads, dim, group)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(kv_len), max(need + [1]) + 1), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.kv = []
        for i, n in enumerate(kv_len):
            k = torch.randn(n, kv_heads, dim, generator=g, device="cuda") * spread
            v = torch.randn(n, kv_heads, dim, generator=g, device="cuda") + 0.5
            slots = self.slots(i, torch.arange(n, device="cuda"))
            qe.qe_cache_append(self.cache, k, v, slots)
            self.kv.append(tuple(x.double() for x in qe.qe_cache_read(self.cache, slots, torch.float32)))
        self.q = torch.randn(sum(q_len), heads, dim, generator=g, device="cuda").to(dtype)
        self.q_start = torch.tensor([0] + list(q_len), device="cuda").cumsum(0).to(torch.int32)
        self.kv_lens = torch.tensor(kv_len, dtype=torch.int32, device="cuda")

    def slots(self, i, j):
        return self.table[i, j // self.cache.page_size].long() * self.cache.page_size + j % self.cache.page_size

    def run(self, **kw):
        q = kw.pop("q", self.q)
        return qe.qe_cache_attention(self.cache, q, self.q_start, self.kv_lens, self.table, kw.pop("max_q", max(self.q_len)),
                                     kw.pop("max_kv", max(self.kv_len)), **kw)

    def plain(self, causal=True, window=0, scale=0.0, q=None):
        """(out, lse, allowed error of out, allowed error of lse), in binary64.

        Rounding that the kernels may do: keys and values to 16 bits once (2^-9 relative; codes times scale), P
        to 16 bits (2^-9), the result to the output type (half an ulp).  A score moves by at most 2^-9 scale
        sum |q k| =: e, a probability by a factor within e^(2 e), so the result by less than
        (e^(2 e) - 1 + 2 (2^-9 + 2^-9)) sum p |v|: the factor 2 covers P's rounding in numerator and sum apart,
        fp32 sums and ex2's 2^-22 vanish beside it."""
        q = self.q if q is None else q
        scale = scale or 1.0 / math.sqrt(self.dim)
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        tol, ltol, at = torch.zeros_like(out), torch.zeros_like(lse), 0
        for n, m, (k, v) in zip(self.q_len, self.kv_len, self.kv):
            rep = self.heads // k.shape[1]
            x = q[at:at + n].double()
            kk, vv = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
            s = torch.einsum("ihd,jhd->hij", x, kk) * scale
            e = (torch.einsum("ihd,jhd->hij", x.abs(), kk.abs()) * scale * 2.0 ** -9).amax(-1) if m else torch.zeros(self.heads, n, dtype=torch.float64, device="cuda")
            pos, j = torch.arange(m - n, m, device="cuda")[:, None], torch.arange(m, device="cuda")
            sees = torch.ones(n, m, dtype=torch.bool, device="cuda")
            if causal:
                sees = j <= pos
                if window:
                    sees &= j > pos - window
            s = s.masked_fill(~sees, -math.inf)
            some = sees.any(-1)
            p = torch.softmax(s, -1).masked_fill(~some[:, None], 0.0)
            out[at:at + n] = torch.einsum("hij,jhd->ihd", p, vv)
            mag = torch.einsum("hij,jhd->ihd", p, vv.abs())
            lse[at:at + n] = torch.logsumexp(s, -1).T if m else -math.inf
            tol[at:at + n] = mag * (torch.expm1(2 * e).T[..., None] + 2.0 ** -7)
            ltol[at:at + n] = e.T + 1e-5
            at += n
        tol += SIZES[q.dtype] * out.abs() + 1e-7
        return out, lse, tol, ltol


def check(b, dtype, **how):
    lse = torch.full(b.q.shape[:2], 7.0, device="cuda")
    got = b.run(lse=lse, **how)
    assert qe.qe_sync_status() == qe.QE_OK
    out, want_lse, tol, ltol = b.plain(**how)
    assert got.dtype == dtype and got.isfinite().all()
    err = (got.double() - out).abs()
    assert (err <= tol).all(), f"largest error {err.max().item():.3g}, {(err / tol).max().item():.2f} of the allowed"
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (got[empty] == 0).all()
    assert ((lse.double() - want_lse)[~empty].abs() <= ltol[~empty]).all()
    # every call gives the same bits, with or without log sums, and with any hint of the longest sequence
    assert torch.equal(got, b.run(**how))
    return got


SHAPES = [(4, 4, 64, 32, 16), (8, 1, 64, 64, 32), (29, 1, 64, 32, 128), (6, 2, 72, 32, 16), (4, 2, 80, 32, 64),
          (3, 3, 96, 32, 32), (8, 2, 128, 32, 64), (16, 1, 128, 64, 16), (5, 5, 128, 128, 256), (4, 1, 8, 64, 16),
          (71, 1, 64, 64, 64)]


@pytest.mark.parametrize("heads,kv_heads,dim,group,page", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_single_tokens(heads, kv_heads, dim, group, page, dtype):
    """One query row per sequence: lengths around the step, the page and the piece, and none at all."""
    kv = [0, 1, 2, 15, 16, 17, 31, 33, 64, 100, 255, 257, 700, 1300]
    b = Batch([1] * len(kv), kv, heads, kv_heads, dim, group, page, dtype, seed=dim)
    check(b, dtype)
    check(b, dtype, causal=False, scale=0.2)


@pytest.mark.parametrize("heads,kv_heads,dim,group,page", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_few_rows(heads, kv_heads, dim, group, page, dtype):
    """Ragged drafts: rows before the first token (more rows than tokens) see nothing; no rows at all are fine."""
    b = Batch([3, 0, 5, 1, 7, 2, 4], [1, 9, 3, 40, 500, 0, 130], heads, kv_heads, dim, group, page, dtype, seed=dim + 1)
    check(b, dtype)
    check(b, dtype, window=7)
    check(b, dtype, window=1)


@pytest.mark.parametrize("heads,kv_heads,dim,group,page", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_chunks_and_prompts(heads, kv_heads, dim, group, page, dtype):
    b = Batch([130, 64, 1, 257], [130, 400, 300, 1030], heads, kv_heads, dim, group, page, dtype, seed=dim + 2)
    check(b, dtype)
    check(b, dtype, window=100)
    check(b, dtype, causal=False)


@pytest.mark.parametrize("spread", [0.01, 8.0])
@pytest.mark.parametrize("q_len", [1, 4, 200])
def test_flat_and_peaked_scores(spread, q_len):
    b = Batch([q_len] * 3, [900, 257, 300], 8, 2, 128, 32, 32, torch.bfloat16, seed=9, spread=spread)
    check(b, torch.bfloat16)


@pytest.mark.parametrize("q_len", [1, 3, 150])
def test_scores_that_grow_and_values_of_many_sizes(q_len):
    """Later tokens score ever higher (the running maximum moves all the time) and hold ever larger or smaller values."""
    for sign in (1.0, -1.0):
        b = Batch([q_len], [640], 4, 2, 128, 64, 64, torch.float16, seed=11)
        j = torch.arange(640, device="cuda")
        g = gen(12)
        k = torch.randn(640, 2, 128, generator=g, device="cuda") * 0.1 + 0.02 * (sign * (j - 320.0))[:, None, None] / 8
        v = torch.randn(640, 2, 128, generator=g, device="cuda") * torch.exp2(sign * (j - 320.0) / 32)[:, None, None]
        qe.qe_cache_append(b.cache, k, v, b.slots(0, j))
        b.kv[0] = tuple(x.double() for x in qe.qe_cache_read(b.cache, b.slots(0, j), torch.float32))
        b.q = b.q.abs()
        check(b, torch.float16)


@pytest.mark.parametrize("q_len", [1, 6, 140])
def test_magnitudes_of_queries(q_len):
    """Query rows of very different sizes, zeros among them."""
    b = Batch([q_len] * 2, [333, 210], 8, 4, 64, 32, 16, torch.bfloat16, seed=13)
    f = torch.exp2(torch.randint(-40, 4, b.q.shape[:2], generator=gen(14), device="cuda").float())
    f[0, :2] = 0.0
    b.q = (b.q.float() * f[..., None]).to(torch.bfloat16)
    check(b, torch.bfloat16)


@pytest.mark.parametrize("q_len,window", [(1, 0), (4, 0), (4, 64), (150, 0), (150, 20)])
def test_a_bad_token_reaches_only_the_rows_that_see_it(q_len, window):
    n = 300
    b = Batch([q_len], [n], 8, 2, 128, 32, 32, torch.bfloat16, seed=15)
    clean = b.run(window=window)
    at = n - 2
    for which in (0, 1):
        k = torch.randn(1, 2, 128, generator=gen(16), device="cuda")
        kv = [k, k.clone()]
        kv[which][0, 1, 5] = math.nan
        j = torch.tensor([at], device="cuda")
        keep = b.cache.data.clone()
        qe.qe_cache_append(b.cache, kv[0], kv[1], b.slots(0, j))
        assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
        got = b.run(window=window)
        pos = torch.arange(n - q_len, n, device="cuda")
        sees = (pos >= at) & ((pos - window < at) if window else torch.ones_like(pos, dtype=torch.bool))
        assert got[sees][:, 4:].isnan().all()                 # the heads of kv head 1
        assert got[:, :4].isfinite().all()
        assert torch.equal(got[~sees], clean[~sees])
        b.cache.data.copy_(keep)
    # a query row that is not finite spoils itself alone
    q = b.q.clone()
    q[0, 3, 9] = math.inf
    got = b.run(window=window, q=q)
    assert got[0, 3].isnan().all()
    got[0, 3], clean[0, 3] = 0, 0
    assert torch.equal(got, clean)


@pytest.mark.parametrize("q_len", [1, 100])
def test_strided_queries_and_outputs(q_len):
    b = Batch([q_len, q_len], [200, 77], 6, 3, 64, 32, 16, torch.float16, seed=17)
    want = b.run()
    n = 2 * q_len
    fused = torch.zeros(n, 6 + 2, 64, dtype=torch.float16, device="cuda")
    fused[:, 1:7] = b.q
    assert torch.equal(b.run(q=fused[:, 1:7]), want)
    odd = torch.zeros(n * 6 * 67 + 1, dtype=torch.float16, device="cuda")[1:].view(n, 6, 67)[..., :64]
    odd.copy_(b.q)
    whole = torch.full((6, n, 69), 7.0, dtype=torch.float16, device="cuda")
    out = whole.permute(1, 0, 2)[..., 3:67]
    assert b.run(q=odd, out=out) is out and torch.equal(out, want)
    assert (whole[..., :3] == 7).all() and (whole[..., 67:] == 7).all()


def test_workspace_streams_and_graphs():
    """A caller's workspace, another stream than the default one, and a captured step replayed on new contents."""
    b = Batch([1] * 3, [3000, 1500, 10], 8, 2, 128, 32, 64, torch.bfloat16, seed=18)
    want = b.run()
    need = qe.qe_cache_attention_workspace(b.cache, 3, 8, 3, 1, 3000)
    assert need > 0
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(b.run(workspace=ws[:need]), want) and (ws[need:] == 0xFF).all()
    with pytest.raises(qe.QEError) as e:
        b.run(workspace=ws[:need - 1])
    assert e.value.status == qe.QE_ERR_OOM
    s = torch.cuda.Stream()
    out = torch.zeros_like(want)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.run(out=out, workspace=ws[:need])
    s.synchronize()
    assert torch.equal(out, want)
    # one decoding step: append, then attend
    k = torch.randn(3, 2, 128, generator=gen(19), device="cuda").to(torch.bfloat16)
    slots = torch.cat([b.slots(i, torch.tensor([n - 1], device="cuda")) for i, n in enumerate(b.kv_len)])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        qe.qe_cache_append(b.cache, k, k, slots)
        b.run(out=out, workspace=ws[:need])
    for _ in range(2):
        k.copy_(torch.randn(k.shape, generator=gen(20), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        qe.qe_cache_append(b.cache, k, k, slots)
        assert torch.equal(b.run(), got)
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("q_len,window,page", [(1, 40, 16), (3, 17, 16), (100, 30, 16), (100, 200, 32)])
def test_pages_that_left_the_window_are_not_looked_up(q_len, window, page):
    n = 900
    b = Batch([q_len, q_len], [n, n - 37], 4, 2, 64, 32, page, torch.bfloat16, seed=30)
    want = b.run(window=window)
    for i, m in enumerate(b.kv_len):
        b.table[i, :(m - q_len - window + 1) // page] = -1        # freed: the oldest row's window starts later
    assert torch.equal(b.run(window=window), want) and qe.qe_sync_status() == qe.QE_OK


def test_device_side_bounds():
    """Page ids out of range, lengths past the table, more rows than announced: reported, nothing read outside."""
    b = Batch([1, 1, 1], [200, 100, 50], 4, 4, 64, 32, 16, torch.bfloat16, seed=21)
    want = b.run()
    keep = b.table.clone()
    b.table[1, 3] = 1 << 30
    got = b.run()
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG
    assert torch.equal(got[[0, 2]], want[[0, 2]]) and got.isfinite().all()
    b.table.copy_(keep)
    b.kv_lens[2] = 1 << 29
    got = b.run()
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG and torch.equal(got[:2], want[:2])
    b.kv_lens[2] = -3
    got = b.run()
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG and torch.equal(got[:2], want[:2]) and (got[2] == 0).all()
    b.kv_lens[2] = 50
    for rows, status in ((3, qe.QE_OK), (2, qe.QE_ERR_INVALID_ARG)):
        q3 = Batch([3], [60], 4, 4, 64, 32, 16, torch.bfloat16, seed=22)
        q3.run(max_q=rows)
        assert qe.qe_sync_status() == status
    assert torch.equal(b.run(), want) and qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("q_len", [1, 40])
def test_offsets_past_32_bits(q_len):
    """A cache of more than 4 GiB, its last pages in use."""
    page, heads, dim = 256, 8, 128
    block = page * heads * (dim + 8 * (dim // 32))
    pages = (5 << 30) // block
    c = qe.KVCache(pages, page, heads, dim, 32)
    n = 600
    table = torch.tensor([[pages - 1, pages - 3, pages - 2]], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    slots = table[0, j // page].long() * page + j % page
    small = Batch([q_len], [n], 16, heads, dim, 32, page, torch.bfloat16, seed=23)
    k, v = (x.float() for x in small.kv[0])
    qe.qe_cache_append(c, k, v, slots)
    qe.qe_cache_append(small.cache, k, v, small.slots(0, j))
    assert torch.equal(qe.qe_cache_read(c, slots, torch.float32)[1], qe.qe_cache_read(small.cache, small.slots(0, j), torch.float32)[1])
    got = qe.qe_cache_attention(c, small.q, small.q_start, small.kv_lens, table, q_len, n)
    assert torch.equal(got, small.run()) and qe.qe_sync_status() == qe.QE_OK


def test_long_context_in_pieces():
    """A context long enough for many pieces, in one page as a cache without paging has it."""
    b = Batch([1, 2], [65535, 40000], 4, 2, 64, 64, 65536, torch.float16, seed=24)
    check(b, torch.float16)


def test_example_runs_end_to_end():
    """The example layer: quantized projections, prompts, then single tokens.  With 8-bit weights what is left is
    mostly the 4-bit keys and values: half a step of a sixteenth of the range each, some 5 per cent of their size."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "quantized_attention.py")
    spec = importlib.util.spec_from_file_location("quantized_attention", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    coarse, fine = mod.run(bits=3), mod.run(bits=8)
    assert fine["prompt"] < 0.2 and fine["step"] < 0.2
    assert fine["prompt"] < coarse["prompt"] and fine["step"] < coarse["step"]
