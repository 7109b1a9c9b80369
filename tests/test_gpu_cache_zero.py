"""Attention over the 4-bit cache where queries, keys or the caller's scale are zero or next to it: every visible token
counts alike, however small the multipliers of the scores get, and masked ones stay out."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.cache_plain import compare
from tests.test_gpu_cache import Batch, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def rewrite(b, key_size):
    """The batch's keys times key_size (0: all zeros) written over the old ones."""
    for i, n in enumerate(b.kv_len):
        if n:
            slots = b.slots(i, torch.arange(n, device="cuda"))
            k, v = (x.float() for x in b.kv[i])
            qe.qe_cache_append(b.cache, k * key_size, v, slots)
            b.kv[i] = tuple(x.double() for x in qe.qe_cache_read(b.cache, slots, torch.float32))


def check(b, **how):
    lse = torch.full(b.q.shape[:2], 7.0, device="cuda")
    got = b.run(lse=lse, **how)
    assert qe.qe_sync_status() == qe.QE_OK
    compare(got, lse, b.q, b.kv, b.q_len, **how)


HOW = [dict(), dict(window=9), dict(causal=False), dict(scale=1e-30), dict(scale=1e-38, window=50)]


@pytest.mark.parametrize("q_len", [1, 4, 40, 200])
@pytest.mark.parametrize("heads,kv_heads,dim,group", [(8, 2, 128, 32), (4, 4, 64, 64), (6, 2, 80, 32), (71, 1, 64, 32)])
@pytest.mark.parametrize("queries,keys", [(0.0, 0.0), (0.0, 2.0 ** -26), (2.0 ** -90, 2.0 ** -40), (1.0, 0.0), (0.0, 1.0)])
def test_small_queries_over_small_keys(q_len, heads, kv_heads, dim, group, queries, keys):
    b = Batch([q_len, q_len], [205, q_len], heads, kv_heads, dim, group, 32, torch.bfloat16, seed=40)
    rewrite(b, keys)
    b.q = (b.q.float() * queries).to(torch.bfloat16)
    for how in HOW:
        check(b, **how)


@pytest.mark.parametrize("q_len", [1, 40])
def test_large_queries_and_scale_over_zero_keys(q_len):
    b = Batch([q_len], [150], 8, 2, 128, 32, 32, torch.bfloat16, seed=43)
    rewrite(b, 0.0)
    b.q = (b.q.float() * 2.0 ** 100).to(torch.bfloat16)
    check(b, scale=1e30)


@pytest.mark.parametrize("q_len", [1, 4, 40, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_zero_rows_among_others(q_len, dtype):
    """Padded rows and padded tokens beside ordinary ones."""
    b = Batch([q_len, 3], [333, 130], 8, 2, 128, 32, 16, dtype, seed=41)
    for i, n in enumerate(b.kv_len):
        j = torch.arange(n, device="cuda")
        zero = (j // 32) % 3 == 1                           # whole steps of zeros, and ordinary ones
        k, v = (x.float() for x in b.kv[i])
        k[zero] = 0.0
        v[(j // 64) % 2 == 1] = 0.0
        qe.qe_cache_append(b.cache, k, v, b.slots(i, j))
        b.kv[i] = tuple(x.double() for x in qe.qe_cache_read(b.cache, b.slots(i, j), torch.float32))
    b.q[torch.rand(b.q.shape[:2], generator=gen(42), device="cuda") < 0.5] = 0.0
    for how in HOW[:3]:
        check(b, **how)
