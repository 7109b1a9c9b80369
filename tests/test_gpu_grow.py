"""Pages, slots and positions from lengths, against a simulation that takes one token after the other."""
import random

import pytest
import torch

from paper_2309_01885_gb300 import build, qe

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


class Books:
    """The state of a batch on the host, and what a call is expected to leave."""

    def __init__(self, seqs, page, pages, width, prefix, rng):
        self.page, self.pages, self.prefix, self.width = page, pages, prefix, width
        order = list(range(pages))
        rng.shuffle(order)
        kept = prefix // page
        self.table = [[-1] * width for _ in range(seqs)]
        for row in self.table:
            row[:kept] = order[:kept]
        free = order[kept:]
        self.first = rng.randrange(pages)
        self.ring = [-7] * pages
        for i, p in enumerate(free):
            self.ring[(self.first + i) % pages] = p
        self.count, self.kv = len(free), [0] * seqs

    def fits(self, new, ends, most):
        P, need, back = self.page, 0, 0
        for b, n in enumerate(new):
            keep = self.prefix if ends[b] else self.kv[b]
            if n < 0 or keep + n > self.width * P:
                return False
            need += -(-(keep + n) // P) - -(-keep // P)
            if ends[b]:
                back += max(0, -(-self.kv[b] // P) - self.prefix // P)
        return sum(new) <= most and need <= self.count and self.count + back <= self.pages

    def step(self, new, ends, most):
        q_start, slots, at, P = [0], [], [], self.page
        if not self.fits(new, ends, most):
            return [0] * (len(new) + 1), [-1] * most, [0] * most
        back = []
        for b, n in enumerate(new):
            if ends[b]:
                back += self.table[b][self.prefix // P:max(self.prefix // P, -(-self.kv[b] // P))]
                self.kv[b] = self.prefix
            for _ in range(n):
                if self.kv[b] % P == 0:
                    self.table[b][self.kv[b] // P] = self.ring[self.first]
                    self.first, self.count = (self.first + 1) % self.pages, self.count - 1
                at.append(self.kv[b])
                slots.append(self.table[b][self.kv[b] // P] * P + self.kv[b] % P)
                self.kv[b] += 1
            q_start.append(len(slots))
        for p in back:
            self.ring[(self.first + self.count) % self.pages] = p
            self.count += 1
        return q_start, slots + [-1] * (most - len(slots)), at + [0] * (most - len(at))

    def on_device(self):
        c = qe.KVCache(self.pages, self.page, 1, 64, 64)
        pool = qe.PagePool(c, ring=torch.tensor(self.ring, dtype=I32, device="cuda"), state=torch.tensor([self.first, self.count], dtype=I32, device="cuda"))
        return c, pool, torch.tensor(self.kv, dtype=I32, device="cuda"), torch.tensor(self.table, dtype=I32, device="cuda")

    def check(self, got, want, kv, pool, table):
        for g, w in zip(got, want):
            assert g.tolist() == w
        assert kv.tolist() == self.kv and table.tolist() == self.table
        assert pool.ring.tolist() == self.ring and pool.state.tolist() == [self.first, self.count]


@pytest.mark.parametrize("seqs,page,prefix,new,most", [
    (1, 16, 0, 1, 1), (1, 16, 0, 40, 50), (3, 16, 32, 7, 30), (64, 64, 0, 1, 64), (64, 16, 48, 1, 70), (33, 32, 0, 100, 4096),
    (257, 16, 16, 30, 9000), (1500, 16, 0, 3, 4096), (2500, 32, 64, 9, 30000), (5, 256, 256, 3000, 16000), (1, 16, 0, 20000, 20001)])
def test_steps(seqs, page, prefix, new, most):
    """A few steps in a row, sequences ending and beginning anew on the way, everything in place."""
    rng = random.Random(seqs * 1000 + page + new)
    width = -(-(4 * new + prefix + 5) // page)
    books = Books(seqs, page, seqs * width + prefix // page + 3, width, prefix, rng)
    cache, pool, kv, table = books.on_device()
    for step in range(4):
        n = [rng.choice((0, 1, new, rng.randint(0, new))) for _ in range(seqs)]
        ends = [step == 0 or rng.random() < 0.2 for _ in range(seqs)]
        while sum(n) > most:
            n[rng.randrange(seqs)] = 0
        want = books.step(n, ends, most)
        got = qe.qe_cache_grow(cache, pool, kv, torch.tensor(n, dtype=I32, device="cuda"), table, most, prefix=prefix,
                               ends=torch.tensor(ends, device="cuda"))
        assert qe.qe_sync_status() == qe.QE_OK
        books.check(got, want, kv, pool, table)


def test_65535_sequences():
    rng = random.Random(1)
    books = Books(65535, 16, 65535 + 21845 + 9, 1, 0, rng)   # pages that come back wait for the next step
    cache, pool, kv, table = books.on_device()
    for ends in (None, [i % 3 == 0 for i in range(65535)]):
        n = [1 + i % 4 for i in range(65535)]
        want = books.step(n, ends or [False] * 65535, sum(n) + 1)
        got = qe.qe_cache_grow(cache, pool, kv, torch.tensor(n, dtype=I32, device="cuda"), table, sum(n) + 1,
                               ends=None if ends is None else torch.tensor(ends, device="cuda"),
                               workspace=torch.empty(qe.qe_cache_grow_workspace(65535), dtype=torch.uint8, device="cuda"))
        assert qe.qe_sync_status() == qe.QE_OK
        books.check(got, want, kv, pool, table)


@pytest.mark.parametrize("most", [60, 6000])
@pytest.mark.parametrize("what", ["negative", "too many tokens", "row too short", "pool empty", "length negative", "length too long", "ring overfull",
                                  "state"])
def test_all_or_nothing(what, most):
    """What does not fit changes nothing and is reported."""
    rng = random.Random(3)
    books = Books(6, 16, 60, 8, 16, rng)
    n, ends = [5, 0, 20, 1, 3, 9], [True] * 6
    books.step(n, ends, most)
    ends = [False, True, False, False, True, False]
    if what == "negative":
        n[3] = -1
    elif what == "too many tokens":
        n = [most // 6 + 1] * 6 if most == 60 else [most, 0, 0, 0, 0, 0]
    elif what == "row too short":
        n[2] = 8 * 16 - books.kv[2] + 1
    elif what == "pool empty":
        books.count = 1
    elif what == "length negative":
        books.kv[5] = -3
    elif what == "length too long":
        books.kv[1] = 8 * 16 + 1
    elif what == "ring overfull":
        books.count, books.kv[4] = 60, 40
    elif what == "state":
        books.first = 60
    cache, pool, kv, table = books.on_device()
    got = qe.qe_cache_grow(cache, pool, kv, torch.tensor(n, dtype=I32, device="cuda"), table, most, prefix=16, ends=torch.tensor(ends, device="cuda"))
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG and qe.qe_sync_status() == qe.QE_OK
    books.check(got, ([0] * 7, [-1] * most, [0] * most), kv, pool, table)


def test_out_of_place_keeps_its_inputs():
    rng = random.Random(5)
    books = Books(9, 16, 100, 10, 0, rng)
    books.step([17] * 9, [True] * 9, 200)
    cache, pool, kv, table = books.on_device()
    was_kv, was_state = kv.clone(), pool.state.clone()
    n, ends = [3, 0, 20, 1, 0, 9, 2, 2, 40], [False, True] + [False] * 7
    want = books.step(n, ends, 100)
    kv_out, state_out = torch.full_like(kv, -9), torch.full_like(pool.state, -9)
    for _ in range(3):                                   # the same step again, from the same state
        got = qe.qe_cache_grow(cache, pool, kv, torch.tensor(n, dtype=I32, device="cuda"), table, 100, ends=torch.tensor(ends, device="cuda"),
                               kv_len_out=kv_out, state_out=state_out)
        assert kv.equal(was_kv) and pool.state.equal(was_state)
        for g, w in zip(got, want):
            assert g.tolist() == w
        assert kv_out.tolist() == books.kv and table.tolist() == books.table and pool.ring.tolist() == books.ring
        assert state_out.tolist() == [books.first, books.count]
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("most", [8, 5000])
def test_captured(most):
    """A captured step keeps its books by itself when it is replayed."""
    rng = random.Random(7)
    books = Books(8, 16, 80, 9, 0, rng)
    cache, pool, kv, table = books.on_device()
    new, ends = torch.ones(8, dtype=I32, device="cuda"), torch.zeros(8, dtype=torch.uint8, device="cuda")
    ws = torch.empty(qe.qe_cache_grow_workspace(8), dtype=torch.uint8, device="cuda")
    args = dict(ends=ends, workspace=ws, q_start=torch.empty(9, dtype=I32, device="cuda"), slots=torch.empty(most, dtype=torch.int64, device="cuda"),
                positions=torch.empty(most, dtype=I32, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = qe.qe_cache_grow(cache, pool, kv, new, table, most, **args)
    for step in range(60):
        over = [step % 13 == b for b in range(8)]
        ends.copy_(torch.tensor(over))
        want = books.step([1] * 8, over, most)
        graph.replay()
        books.check(got, want, kv, pool, table)
    assert qe.qe_sync_status() == qe.QE_OK


def test_on_another_stream():
    rng = random.Random(9)
    books = Books(40, 16, 300, 7, 0, rng)
    cache, pool, kv, table = books.on_device()
    new = torch.full((40,), 13, dtype=I32, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = qe.qe_cache_grow(cache, pool, kv, new, table, 5000, stream=s)
    s.synchronize()
    books.check(got, books.step([13] * 40, [False] * 40, 5000), kv, pool, table)
