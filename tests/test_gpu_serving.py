"""Steps of a serving loop: pages and slots for new tokens, projections on quantized weights, norms and rotation, the 4-bit
cache and attention behind a shared prefix, as one run.  Each stage is held against binary64 on what the stage before it left,
within that operator's own bounds; keys and values are what the cache held right after they were written, so that a page handed
out twice, or taken back too early, is seen."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests import cache_plain, test_gpu_linear as products, test_gpu_rotate as rotations

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def integers(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Block:
    """An attention layer and the two products behind it, every weight quantized."""

    def __init__(self, dtype, bits, prefix, seqs, width=264, heads=6, kv_heads=2, dim=64, page=16, pages=64, group=0, seed=0):
        g = products.gen(seed)
        self.dtype, self.prefix, self.heads, self.kv_heads, self.dim, self.page = dtype, prefix, heads, kv_heads, dim, page
        self.w, self.w64 = {}, {}
        for i, (name, q, p) in enumerate((("qkv", (heads + 2 * kv_heads) * dim, width), ("o", width, heads * dim),
                                          ("up", 2 * width, width), ("down", width, 2 * width))):
            grids = products.layer(q, p, bits, group, seed + i)
            self.w[name] = qe.QuantizedWeights(*grids, bits, group_size=group)
            self.w64[name] = products.weights64(*grids, group)
        self.bias = torch.randn((heads + 2 * kv_heads) * dim, generator=g, device="cuda").mul_(0.1).to(dtype)
        self.q_norm, self.k_norm = ((1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).to(dtype) for _ in range(2))
        self.rope = qe.Rope(dim, theta=10000.0)
        self.freq = [10000.0 ** (-2.0 * i / dim) for i in range(dim // 2)]
        self.cache = qe.KVCache(pages, page, kv_heads, dim)
        self.cache.data.fill_(0xFF)                      # grids that are never written are NaN
        self.pool = qe.PagePool(self.cache)
        self.prefix_table = torch.full((1, max(1, prefix // page)), -1, dtype=torch.int32, device="cuda")
        self.table = torch.full((seqs, 12), -1, dtype=torch.int32, device="cuda")
        self.kv_len = integers([prefix] * seqs)

    def step(self, x, table, kv_len, new, prefix, max_q, max_kv, ends=None):
        c, h, kv = self.cache, self.heads, self.kv_heads
        start, slots, positions = qe.qe_cache_grow(c, self.pool, kv_len, new, table, x.shape[0], ends=ends, prefix=prefix)
        y = qe.qe_linear(self.w["qkv"], x, bias=self.bias)
        heads = y.unflatten(-1, (h + 2 * kv, self.dim))
        v = heads[:, h + kv:]
        q, k = qe.qe_norm_rotate(heads[:, :h], heads[:, h:h + kv], positions, self.rope, q_weight=self.q_norm, k_weight=self.k_norm)
        qe.qe_cache_append(c, k, v, slots)
        a = qe.qe_cache_attention_shared(c, q, start, kv_len, table, max_q, max_kv, self.prefix_table[0], prefix)
        o = qe.qe_linear(self.w["o"], a.flatten(1), residual=x)
        up = qe.qe_linear(self.w["up"], o, activation="silu")
        return dict(start=start, slots=slots, positions=positions, y=y, heads=heads, q=q, k=k, a=a, o=o, up=up,
                    out=qe.qe_linear(self.w["down"], up, residual=o))

    def check(self, r, x, new, before, behind):
        """before: tokens in front of each sequence's new ones; behind: the (keys, values) there.  Returns those with the new ones."""
        assert qe.qe_sync_status() == qe.QE_OK
        n, h, kv = sum(new), self.heads, self.kv_heads
        assert r["start"].tolist() == [sum(new[:b]) for b in range(len(new) + 1)]
        assert r["positions"][:n].tolist() == [l + i for l, m in zip(before, new) for i in range(m)]
        live, x = {name: t[:n] for name, t in r.items()}, x[:n]
        products.check(live["y"], self.w64["qkv"], x, bias=self.bias)
        for got, part, w in ((live["q"], slice(0, h), self.q_norm), (live["k"], slice(h, h + kv), self.k_norm)):
            rotations.check(got, live["heads"][:, part], live["positions"], self.freq, False, w, 1e-6)
        kr, vr = (t.double() for t in qe.qe_cache_read(self.cache, live["slots"], torch.float32))
        seen, at = [], 0
        for (k0, v0), m in zip(behind, new):
            seen.append((torch.cat([k0, kr[at:at + m]]), torch.cat([v0, vr[at:at + m]])))
            at += m
        want, _, tol, _ = cache_plain.plain(live["q"], seen, new)
        err = (live["a"].double() - want).abs()
        assert (err <= tol).all(), f"up to {(err / tol).max().item():.2f} of the allowed"
        products.check(live["o"], self.w64["o"], live["a"].flatten(1), residual=x)
        products.check(live["up"], self.w64["up"], live["o"], act="silu")
        products.check(live["out"], self.w64["down"], live["up"], residual=live["o"])
        return seen


def begun(block, g, width):
    """The prefix goes through the layer as a sequence of its own; its keys and values."""
    none = torch.zeros(0, block.kv_heads, block.dim, dtype=torch.float64, device="cuda")
    if not block.prefix:
        return none, none
    x = torch.randn(block.prefix, width, generator=g, device="cuda").to(block.dtype)
    r = block.step(x, block.prefix_table, integers([0]), integers([block.prefix]), 0, block.prefix, block.prefix)
    return block.check(r, x, [block.prefix], [0], [(none, none)])[0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits,group,prefix", [(4, 0, 48), (3, 128, 32), (8, 64, 0)])
def test_steps_of_a_batch(dtype, bits, group, prefix):
    width, g = 264, products.gen(bits)
    block = Block(dtype, bits, prefix, 5, width, group=group, seed=10 * bits)
    first = begun(block, g, width)
    seen, lens = [first] * 5, [prefix] * 5
    steps = [([3, 1, 0, 20, 40], None), ([1] * 5, None), ([1, 1, 1, 1, 0], [0, 0, 0, 0, 1]), ([1, 9, 1, 1, 30], [0, 1, 0, 1, 0]),
             ([1] * 5, None), ([17, 1, 1, 1, 1], [1, 0, 1, 0, 0]), ([0] * 5, [1] * 5), ([2, 70, 2, 2, 2], None), ([1] * 5, None)]
    for new, ends in steps:
        for b in range(5):
            if ends and ends[b]:
                seen[b], lens[b] = first, prefix
        pad = sum(new) + 3                               # rows behind the last token are of no sequence
        x = torch.randn(pad, width, generator=g, device="cuda").to(dtype)
        at = None if ends is None else torch.tensor(ends, dtype=torch.uint8, device="cuda")
        longest = max(a + b for a, b in zip(lens, new))
        r = block.step(x, block.table, block.kv_len, integers(new), prefix, max(max(new), 1), longest, at)
        assert (r["slots"][sum(new):] == -1).all()
        seen = block.check(r, x, new, lens, seen)
        lens = [a + b for a, b in zip(lens, new)]
        assert block.kv_len.tolist() == lens


def test_a_captured_step_advances_as_an_eager_one():
    """Two graphs of one state, replayed in turn, against the same steps made eagerly, bit by bit."""
    width, g = 264, products.gen(3)
    block = Block(torch.bfloat16, 4, 32, 4, width, seed=5)
    begun(block, g, width)
    state = [block.cache.data, block.pool.ring, block.pool.state, block.table, block.kv_len]
    held = [t.clone() for t in state]
    x, ends = torch.zeros(4, width, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, dtype=torch.uint8, device="cuda")
    new = integers([1] * 4)
    inputs = [(torch.randn(4, width, generator=g, device="cuda").to(torch.bfloat16), torch.tensor(e, dtype=torch.uint8, device="cuda"))
              for e in ([0] * 4, [0, 1, 0, 0], [0] * 4, [1, 0, 0, 1], [0] * 4, [0] * 4)]

    def run():
        return block.step(x, block.table, block.kv_len, new, 32, 1, 100, ends)["out"]

    want = []
    for rows, over in inputs:
        x.copy_(rows), ends.copy_(over)
        want.append(run().clone())
    assert qe.qe_sync_status() == qe.QE_OK
    after = [t.clone() for t in state]
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for t, was in zip(state, held):
        t.copy_(was)
    for i, (rows, over) in enumerate(inputs):
        x.copy_(rows), ends.copy_(over)
        graph, out = graphs[i % 2]
        graph.replay()
        assert torch.equal(out, want[i])
    assert all(torch.equal(t, was) for t, was in zip(state, after))
    assert qe.qe_sync_status() == qe.QE_OK


def test_two_streams_at_once():
    """Two batches on two streams, their launches in turn with nothing in between to wait for, against one after the other."""
    width = 264

    def made():
        blocks, rows = [], []
        for seed in (21, 22):
            g = products.gen(seed)
            block = Block(torch.bfloat16, 4, 32, 4, width, seed=seed)
            begun(block, g, width)
            blocks.append(block)
            rows.append([torch.randn(n, width, generator=g, device="cuda").to(torch.bfloat16) for n in (4, 4, 80, 4, 160, 4)])
        return blocks, rows

    def step(block, x):
        n = x.shape[0] // 4
        return block.step(x, block.table, block.kv_len, n_of[n], 32, n, 200)["out"]

    n_of = {n: integers([n] * 4) for n in (1, 20, 40)}
    blocks, rows = made()
    want = [[step(block, x) for x in xs] for block, xs in zip(blocks, rows)]
    torch.cuda.synchronize()
    blocks, rows = made()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for i in range(6):
        for b in range(2):
            with torch.cuda.stream(streams[b]):
                got[b].append(step(blocks[b], rows[b][i]))
    torch.cuda.synchronize()
    assert qe.qe_sync_status() == qe.QE_OK
    assert all(torch.equal(x, y) for b in range(2) for x, y in zip(got[b], want[b]))
