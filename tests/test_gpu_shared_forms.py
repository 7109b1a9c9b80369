"""Attention behind a shared prefix in all of its forms (few rows and tiles, bf16 and fp16): tokens and queries that are not finite,
pages out of range, batches without a mask (bounds: tests/cache_plain.py)."""
import math

import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests import cache_plain
from tests.test_gpu_shared import Batch

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def shape(n, prefix):
    """Two sequences behind the prefix with n rows each, an idle place, and one that does not reach past the prefix."""
    return [(n, prefix + n + 60), (n, prefix + n), (0, prefix), (min(n, prefix - 5), prefix - 5)]


def slot(row, j, page):
    return (row[j // page].long() * page + j % page)[None]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,group", [(64, 64), (128, 32), (96, 32)])
@pytest.mark.parametrize("n,prefix", [(1, 100), (40, 100), (40, 1500), (150, 300)])
def test_bad_tokens_reach_only_rows_that_see_them(n, prefix, dim, group, dtype):
    """A key or value that is not finite, of kv head 1: in the prefix, of a sequence's own, of the place that has all of its own."""
    b = Batch(shape(n, prefix), prefix, 8, 2, dim, group, page=16, dtype=dtype, seed=n + prefix)
    clean = b.check()
    clean_data = b.cache.data.clone()
    seq = torch.tensor([i for i, m in enumerate(b.q_len) for _ in range(m)], device="cuda")
    pos = torch.cat([torch.arange(b.kv[i][0].shape[0] - m, b.kv[i][0].shape[0], device="cuda") for i, m in enumerate(b.q_len)])
    own = prefix + 30 + n // 2
    for which in (0, 1):
        for where, sees in ((slot(b.prefix_pages, prefix - 3, 16), seq < 2), (slot(b.table[0], own, 16), (seq == 0) & (pos >= own)),
                            (slot(b.table[3], prefix // 2, 16), (seq == 3) & (pos >= prefix // 2))):
            kv = [torch.randn(1, 2, dim, device="cuda") for _ in range(2)]
            kv[which][0, 1, 5] = math.nan
            good = [t.clone() for t in kv]
            good[which][0, 1, 5] = 0.0
            qe.qe_cache_append(b.cache, *kv, where)
            assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
            got = b.attend()
            assert got[sees][:, 4:].isnan().all() and got[sees][:, :4].isfinite().all()
            assert got[~sees].equal(clean[~sees])
            qe.qe_cache_append(b.cache, *good, where)             # the same token without it: kv head 0 sees no difference
            assert got[:, :4].equal(b.attend()[:, :4])
            b.cache.data.copy_(clean_data)
    assert b.attend().equal(clean) and qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,prefix", [(1, 100), (40, 100), (40, 1500), (150, 300)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_queries_that_are_not_finite_stay_in_their_row(n, prefix, value, dtype):
    b = Batch(shape(n, prefix), prefix, 8, 2, 64, 32, page=16, dtype=dtype, seed=n + prefix + 1)
    clean = b.check()
    rows = [(0, 3), (n - 1, 0), (n, 7), (2 * n - 1, 4)]
    for r, h in rows:
        b.q[r, h, 9] = value
    got = b.attend()
    assert qe.qe_sync_status() == qe.QE_OK
    for r, h in rows:
        assert got[r, h].isnan().all()
        got[r, h], clean[r, h] = 0, 0
    assert got.equal(clean)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,prefix", [(1, 100), (40, 100), (40, 1500), (150, 300)])
@pytest.mark.parametrize("page_id", [1 << 20, -1])
def test_bad_pages_count_as_not_there(n, prefix, page_id, dtype):
    """A page of the prefix out of range, one of a sequence's own, and both."""
    for bad_prefix, bad_own in ((True, False), (False, True), (True, True)):
        b = Batch(shape(n, prefix), prefix, 8, 2, 64, 32, page=16, dtype=dtype, seed=n + prefix + 2)
        of_prefix, of_own = 2, (prefix + 20) // 16 + 1
        gone = [set(), set(), set(), set()]
        if bad_prefix:
            b.prefix_pages[of_prefix] = page_id
            for i in range(2):
                gone[i] |= set(range(of_prefix * 16, of_prefix * 16 + 16))
        if bad_own:
            b.table[0, of_own] = page_id
            gone[0] |= set(range(of_own * 16, of_own * 16 + 16))
        lse = torch.empty(b.q.shape[:2], device="cuda")
        out = b.attend(lse=lse)
        assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG
        # positions stay what they were, so each row is compared as a sequence of its own
        at = 0
        for i, m in enumerate(b.q_len):
            k, v = b.kv[i]
            total = k.shape[0]
            for r in range(m):
                if r % 13 == 0 or r + 1 == m:
                    keep = [j for j in range(total - m + r + 1) if j not in gone[i]]
                    cache_plain.compare(out[at:at + 1], lse[at:at + 1], b.q[at:at + 1], [(k[keep], v[keep])], [1], causal=False)
                at += 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,dim,group", [(8, 2, 64, 32), (6, 2, 80, 32), (4, 1, 128, 128)])
@pytest.mark.parametrize("prefix,batch", [(20, [(1, 20), (1, 25), (3, 19), (1, 0), (2, 100)]), (300, [(100, 300), (50, 900), (60, 299), (0, 400)]),
                                          (2000, [(33, 2000), (70, 2100)])])
def test_without_a_mask(prefix, batch, heads, kv_heads, dim, group, dtype):
    b = Batch(batch, prefix, heads, kv_heads, dim, group, dtype=dtype, causal=False, seed=prefix)
    want = b.check()
    assert b.attend().equal(want)
