"""The workspace that attention over the 4-bit cache asks for does for every smaller batch too: a program takes it once,
for its largest one.  The launches go to a runtime that runs none."""
import random

import pytest

from paper_2309_01885_gb300 import qe
from tests import cache_host as host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host.load(tmp_path_factory.mktemp("host"))


def test_one_sequence_after_nineteen(lib):
    c = host.cache(8, 128, 32)
    big = host.workspace(lib, c, host.batch(19, 200, 8000, 32))
    one = host.batch(1, 200, 8000, 32)
    assert host.workspace(lib, c, one) <= big
    assert host.attend(lib, c, one, 0x100000, big) == qe.QE_OK


@pytest.mark.parametrize("seed", range(40))
def test_enough_for_every_smaller_batch(lib, seed):
    rng = random.Random(seed)
    kv_heads = rng.choice((1, 2, 3, 8, 32, 200))
    dim, group = rng.choice(((64, 32), (64, 64), (80, 32), (96, 32), (128, 32), (128, 128)))
    q_heads = kv_heads * rng.choice((1, 1, 4, 7, 29, 71))
    c = host.cache(kv_heads, dim, group)

    def up_to(n):
        return int(round(n ** rng.random()))

    for _ in range(50):
        seqs, q, kv = up_to(300), up_to(4000), up_to(200000)
        most = host.workspace(lib, c, host.batch(seqs, q, kv, q_heads, rows=q))
        for _ in range(20):
            s, n, m = up_to(seqs), up_to(q), up_to(kv)
            at = host.batch(s, n, m, q_heads, rows=n, window=rng.choice((0, up_to(m))))
            assert host.workspace(lib, c, at) <= most, (seqs, q, kv, s, n, m)
            assert host.attend(lib, c, at, 0x100000, most) == qe.QE_OK, (seqs, q, kv, s, n, m, at.window)
