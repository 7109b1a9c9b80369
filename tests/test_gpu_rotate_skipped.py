"""Tokens that norms and rotation pass over: those with a negative position (bounds: tests/test_gpu_rotate.py)."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.test_gpu_rotate import check, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def batch(tokens, dtype):
    g = gen(tokens)
    q, k = (torch.randn(tokens, n, 64, generator=g, device="cuda").to(dtype) for n in (5, 2))
    pos = torch.randint(-5, 10, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = -1
    return q, k, pos, (1 + torch.randn(64, generator=g, device="cuda")).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [1, 6, 1500, 5000])
def test_norms_without_a_rotation(tokens, dtype):
    q, k, pos, w = batch(tokens, dtype)
    out = [torch.full_like(x, 7.0) for x in (q, k)]
    qe.qe_norm_rotate(q, k, pos, None, q_weight=w, k_weight=w, q_out=out[0], k_out=out[1])
    on = pos >= 0
    for x, y in zip((q, k), out):
        assert (y[~on] == 7.0).all()
        check(y[on], x[on], pos[on], None, False, w, 1e-6)
    assert qe.qe_sync_status() == qe.QE_OK
