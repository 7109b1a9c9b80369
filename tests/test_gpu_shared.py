"""Attention over a prefix that sequences share and their own tokens, against binary64 (tests/cache_plain.py's bounds)."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests import cache_plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


class Batch:
    """Sequences of (query rows, cached tokens) behind a prefix; those that do not reach past it have pages of their own."""

    def __init__(self, shape, prefix, heads=8, kv_heads=2, dim=64, group=32, page=16, dtype=torch.bfloat16, causal=True, seed=0, gap=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.prefix, self.causal, self.page = prefix, causal, page
        q_len, kv_len = [n for n, _ in shape], [m for _, m in shape]
        joins = [m - (n if causal else 0) >= prefix for n, m in shape]
        full = -(-prefix // page)
        need = [max(0, -(-m // page) - prefix // page) if j else -(-m // page) for m, j in zip(kv_len, joins)]
        pages = full + sum(need) + 1
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
        width = max([1] + [-(-m // page) for m in kv_len])
        table, at = torch.full((len(shape), width), -1, dtype=torch.int32), full   # prefix pages in a table are not looked at
        for b, n in enumerate(need):
            first = prefix // page if joins[b] else 0
            table[b, first:first + n] = order[at:at + n]
            at += n
        self.cache = qe.KVCache(pages, page, kv_heads, dim, group)
        self.cache.data.fill_(0xFF)                      # grids that are never written are NaN
        self.prefix_pages, self.table = order[:full].cuda(), table.cuda()

        def write(row, lo, hi):
            j = torch.arange(lo, hi, device="cuda")
            slots = row[j // page].long() * page + j % page
            k, v = (torch.randn(hi - lo, kv_heads, dim, generator=g, device="cuda") for _ in range(2))
            if hi > lo:
                qe.qe_cache_append(self.cache, k, v, slots)
            return qe.qe_cache_read(self.cache, slots, torch.float32)

        k0, v0 = write(self.prefix_pages, 0, prefix)
        self.kv = []
        for b, m in enumerate(kv_len):
            k, v = write(self.table[b], prefix if joins[b] else 0, m)
            self.kv.append((torch.cat([k0, k]).double(), torch.cat([v0, v]).double()) if joins[b] else (k.double(), v.double()))
        self.q_len, rows = q_len, sum(q_len)
        self.q = torch.randn(rows + 2 * gap, heads, dim, generator=g, device="cuda").mul_(1.5).to(dtype)
        self.gap, self.rows = gap, rows
        self.start = (torch.tensor([0] + q_len, device="cuda").cumsum(0) + gap).to(torch.int32)
        self.kv_len = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
        self.max_q, self.max_kv = max(q_len), max(kv_len)

    def attend(self, **kw):
        return qe.qe_cache_attention_shared(self.cache, self.q, self.start, self.kv_len, self.table, self.max_q, self.max_kv,
                                            self.prefix_pages, self.prefix, causal=self.causal, **kw)

    def check(self, **kw):
        lse = torch.full(self.q.shape[:2], 3.0, dtype=torch.float32, device="cuda")
        out = torch.full_like(self.q, 3.0)
        self.attend(out=out, lse=lse, **kw)
        assert qe.qe_sync_status() == qe.QE_OK
        own = slice(self.gap, self.gap + self.rows)
        cache_plain.compare(out[own], lse[own], self.q[own], self.kv, self.q_len, causal=self.causal)
        for part in (out[:self.gap], out[self.gap + self.rows:], lse[:self.gap], lse[self.gap + self.rows:]):
            assert (part == 3.0).all()                   # rows of no sequence
        return out


SHAPES = [
    (1, [(1, 2)]), (16, [(1, 17), (1, 40)]), (5, [(1, 6), (1, 9), (1, 100)]), (100, [(1, 101), (1, 300), (1, 0), (1, 150)]),
    (100, [(1, 100), (1, 101), (1, 99), (1, 1), (2, 102), (2, 101), (3, 101)]),       # at, behind and inside the prefix
    (37, [(5, 42), (7, 90), (3, 38), (1, 2), (4, 4)]), (64, [(1, 65 + 3 * i) for i in range(40)]), (700, [(1, 701 + i % 5) for i in range(70)]),
    (3000, [(1, 3001), (1, 3500), (1, 10)]), (300, [(40, 340), (70, 500), (1, 301), (20, 20)]), (1000, [(33, 1033 + 50 * i) for i in range(9)]),
    (129, [(200, 400), (1, 0), (3, 200)]), (4100, [(9, 4109), (9, 4200)]), (20000, [(1, 20001), (2, 20500)]), (50, [(1, 4000), (1, 52)])]


@pytest.mark.parametrize("prefix,shape", SHAPES)
@pytest.mark.parametrize("heads,kv_heads,dim,group", [(8, 2, 64, 32), (4, 4, 128, 64), (29, 1, 64, 64), (6, 2, 80, 32), (12, 2, 128, 128)])
def test_against_binary64(prefix, shape, heads, kv_heads, dim, group):
    i = prefix + heads
    Batch(shape, prefix, heads, kv_heads, dim, group, page=(16, 32, 64)[i % 3], dtype=(torch.bfloat16, torch.float16)[i % 2], seed=i).check()


@pytest.mark.parametrize("prefix,shape", [(20, [(1, 20), (1, 25), (3, 19), (1, 0), (2, 100)]), (300, [(100, 300), (50, 900), (60, 299)])])
def test_not_causal(prefix, shape):
    Batch(shape, prefix, causal=False, seed=1).check()


@pytest.mark.parametrize("prefix,shape", SHAPES[2:6] + SHAPES[9:11])
def test_rows_of_no_sequence_and_workspaces(prefix, shape):
    b = Batch(shape, prefix, seed=2, gap=3)
    want = b.check()
    n = qe.qe_cache_attention_shared_workspace(b.cache, len(shape), 8, b.q.shape[0], b.max_q, b.max_kv, prefix)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    assert b.check(workspace=ws).equal(want)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(qe.QEError) as e:
        b.attend(workspace=small)
    assert e.value.status == qe.QE_ERR_OOM


def test_strided_queries_and_results():
    b = Batch([(1, 130), (2, 300), (1, 101)], 100, seed=3)
    want = b.attend()
    fused = torch.zeros(b.rows, 12, 64, dtype=b.q.dtype, device="cuda")
    fused[:, 2:10] = b.q
    out = torch.zeros(b.rows, 9, 68, dtype=b.q.dtype, device="cuda")
    b.q = fused[:, 2:10]
    b.attend(out=out[:, :8, :64])
    assert out[:, :8, :64].equal(want) and (out[:, 8:] == 0).all() and (out[..., 64:] == 0).all()


def test_no_prefix_is_plain_attention():
    b = Batch([(1, 30), (3, 70)], 0, seed=4)
    plain = qe.qe_cache_attention(b.cache, b.q, b.start, b.kv_len, b.table, b.max_q, b.max_kv)
    assert b.attend().equal(plain)
    b.check()


def test_bad_pages_are_reported():
    """A prefix page out of range: its tokens count as not there, for every sequence; a sequence's own, for it alone."""
    b = Batch([(1, 70), (1, 90), (1, 101)], 64, seed=5)
    b.prefix_pages[1] = 1 << 20
    keep = [j for j in range(64) if not 16 <= j < 32]
    b.kv = [(torch.cat([k[keep], k[64:]]), torch.cat([v[keep], v[64:]])) for k, v in b.kv]
    lse = torch.empty(3, 8, device="cuda")
    out = b.attend(lse=lse)
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG
    cache_plain.compare(out, lse, b.q, b.kv, b.q_len)


def test_tokens_that_are_not_finite():
    """A bad token in the prefix is seen by every sequence behind it, one of a sequence's own by that one."""
    b = Batch([(1, 70), (1, 90), (1, 10)], 64, seed=6)
    want = b.attend()
    bad = torch.full((1, 2, 64), float("nan"), device="cuda")
    qe.qe_cache_append(b.cache, bad, bad, (b.table[1, 80 // 16].long() * 16 + 80 % 16)[None])
    assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
    got = b.attend()
    assert got[0].equal(want[0]) and got[1].isnan().all() and got[2].equal(want[2])
    qe.qe_cache_append(b.cache, bad, bad, (b.prefix_pages[2].long() * 16 + 3)[None])
    assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
    got = b.attend()
    assert got[:2].isnan().all() and got[2].equal(want[2])


def test_two_captured_graphs_and_a_stream():
    """Graphs captured with a workspace of their own each, replayed after the lengths have changed."""
    b = Batch([(1, 150), (1, 120), (1, 101)], 100, seed=7)
    ws = [torch.empty(qe.qe_cache_attention_shared_workspace(b.cache, 3, 8, 3, 1, b.max_kv, 100), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.empty_like(b.q) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, w, o in zip(graphs, ws, out):
        with torch.cuda.graph(g):
            b.attend(out=o, workspace=w)
    full = b.attend()
    b.kv_len.copy_(torch.tensor([140, 101, 0], dtype=torch.int32))
    for g in graphs:
        g.replay()
    want = b.attend()
    assert out[0].equal(want) and out[1].equal(want) and not want.equal(full) and (want[2] == 0).all()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = b.attend(stream=s)
    s.synchronize()
    assert got.equal(want)


@pytest.mark.parametrize("max_kv", [0, 1, 50, 3000, 1 << 20])
@pytest.mark.parametrize("shape", [[(1, 101), (1, 300), (1, 0), (1, 150)], [(40, 150), (33, 400)]])
def test_the_longest_sequence_only_plans_the_work(shape, max_kv):
    """max_kv below the prefix, below what is there, or far above it."""
    b = Batch(shape, 100, seed=31)
    b.max_kv = max_kv
    b.check()
