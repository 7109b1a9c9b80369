"""Attention over the 4-bit cache in each form that a call may be cut into: steps dealt out over one wave and joined by
item or by border, a CTA of four or eight warps for each item, tiles whole and in pieces; with 1, 2 and 4 row tiles, all
head dims, both types; and with any hint of the longest sequence.  All against binary64."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.cache_plain import compare
from tests.test_gpu_cache import Batch

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def check(b, max_kv=None, **how):
    lse = torch.full(b.q.shape[:2], 7.0, device="cuda")
    hint = {} if max_kv is None else dict(max_kv=max_kv)
    got = b.run(lse=lse, **hint, **how)
    assert qe.qe_sync_status() == qe.QE_OK
    compare(got, lse, b.q, b.kv, b.q_len, **how)
    assert torch.equal(got, b.run(**hint, **how))        # the same bits each time
    return got


# (query heads, kv heads, dim, group), query rows: 1, 2 and 4 tiles of 8 pairs; the last of each dim in two items a head
FEW = [((8, 2, 64, 32), 1), ((8, 2, 64, 64), 4), ((8, 2, 64, 32), 8), ((29, 1, 64, 64), 1),
       ((6, 2, 80, 32), 1), ((6, 2, 96, 32), 5), ((6, 2, 96, 32), 8),
       ((8, 2, 128, 32), 1), ((8, 2, 128, 64), 2), ((8, 2, 128, 128), 4), ((8, 2, 128, 32), 6)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape,q", FEW)
def test_steps_dealt_out_few_items(shape, q, dtype):
    """Contexts above 2048 tokens, fewer items than workers: items are cut, and joined one by one."""
    heads, kv_heads, dim, group = shape
    b = Batch([q, q, 0, q, q], [3000, 2100, 9, 0, 2600], heads, kv_heads, dim, group, 64, dtype, seed=80)
    check(b)
    check(b, window=2500)
    check(b, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads,dim,group,q", [(32, 32, 64, 32, 1), (64, 32, 64, 64, 6), (64, 32, 64, 32, 16), (32, 32, 80, 32, 1),
                                                        (32, 32, 96, 32, 11), (64, 32, 128, 128, 2), (32, 32, 128, 32, 16)])
def test_steps_dealt_out_many_items(heads, kv_heads, dim, group, q, dtype):
    """More items than workers (1216 at most): joined at the borders of the workers; empty sequences in between."""
    kv = [(37 * i * i + 11 * i) % 331 for i in range(60)]
    rows = [0 if i % 7 == 3 else 1 + i % q for i in range(60)]
    kv[5] = kv[6] = kv[30] = 0
    rows[59] = q
    b = Batch(rows, kv, heads, kv_heads, dim, group, 16, dtype, seed=81)
    assert 60 * kv_heads > 1216
    check(b)
    check(b, window=40)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape,q", FEW)
def test_a_cta_for_each_item(shape, q, dtype):
    """Short contexts: up to 152 items with eight warps each, up to 1216 with four."""
    heads, kv_heads, dim, group = shape
    for seqs in (3, 140):
        kv = [(i * 271 + 5) % 1050 if i % 5 else i % 3 for i in range(seqs)]
        b = Batch([q] * seqs, kv, heads, kv_heads, dim, group, 32, dtype, seed=82)
        check(b)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape,q", [((8, 2, 128, 32), 40), ((6, 2, 80, 32), 50), ((71, 1, 64, 64), 1), ((5, 1, 128, 128), 103)])
def test_tiles_in_pieces(shape, q, dtype):
    heads, kv_heads, dim, group = shape
    b = Batch([q, 1, q], [9000, 700, 4097], heads, kv_heads, dim, group, 64, dtype, seed=83)
    check(b)
    check(b, window=3000)
    check(b, causal=False)


@pytest.mark.parametrize("shape,q", [((8, 2, 128, 32), 1), ((8, 2, 64, 32), 8), ((6, 2, 96, 32), 5), ((8, 2, 128, 64), 60)])
def test_any_hint_of_the_longest_sequence(shape, q):
    """max_kv plans the work, right or not: results differ by rounding at most."""
    heads, kv_heads, dim, group = shape
    b = Batch([q, q, q], [2900, 130, 1500], heads, kv_heads, dim, group, 32, BF16, seed=84)
    for hint in (0, 1, 33, 1000, 2100, 2900, 5000, 1 << 17, 1 << 30):
        check(b, max_kv=hint)
        check(b, max_kv=hint, window=700)


@pytest.mark.parametrize("hint", [0, 50, 5000, 1 << 30])
def test_any_hint_with_many_items(hint):
    kv = [(53 * i) % 290 for i in range(45)]
    b = Batch([1] * 45, kv, 32, 32, 64, 32, 16, F16, seed=85)
    check(b, max_kv=hint)
