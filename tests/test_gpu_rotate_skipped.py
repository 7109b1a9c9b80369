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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rope", [dict(rotary_dim=64), dict(rotary_dim=64, interleaved=True), dict(rotary_dim=24), dict(rotary_dim=20), None], ids=str)
@pytest.mark.parametrize("tokens", [3, 1500, 5000])
def test_results_that_are_allocated_hold_zeros(tokens, rope, dtype):
    """A padded batch's results do not depend on what the memory held; those of the caller's stay."""
    q, k, pos, w = batch(tokens, dtype)
    n = 0 if rope is None else rope["rotary_dim"]
    freq = [10000.0 ** (-2.0 * i / n) for i in range(n // 2)] if rope else None
    how = (freq, bool(rope and rope.get("interleaved")), w, 1e-6)
    rope, on = qe.Rope(**rope) if rope else None, pos >= 0
    for kw in ({}, dict(q_out=torch.full_like(q, 7.0)), dict(k_out=torch.full_like(k, 7.0))):
        junk = [torch.full_like(x, float("nan")) for x in (q, k)]
        del junk                                          # (the allocator hands its memory out again)
        got = qe.qe_norm_rotate(q, k, pos, rope, q_weight=w, k_weight=w, **kw)
        for name, x, y in zip(("q_out", "k_out"), (q, k), got):
            assert (y[~on] == (7.0 if name in kw else 0.0)).all()
            check(y[on], x[on], pos[on], *how)
    got = qe.qe_norm_rotate(None, k, pos, rope, k_weight=w)[1]
    assert (got[~on] == 0).all()
    check(got[on], k[on], pos[on], *how)
    assert qe.qe_sync_status() == qe.QE_OK
