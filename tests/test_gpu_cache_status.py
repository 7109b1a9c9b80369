"""Errors that the device latches: one does not hide another."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("slot,value,want", [
    (3, 1.0, []), (99, 1.0, [qe.QE_ERR_INVALID_ARG]), (3, float("nan"), [qe.QE_ERR_NUMERIC]),
    (99, float("nan"), [qe.QE_ERR_INVALID_ARG, qe.QE_ERR_NUMERIC])])
def test_each_error_is_reported(slot, value, want):
    c = qe.KVCache(2, 16, 1, 64, 32)
    x = torch.randn(2, 1, 64, generator=torch.Generator(device="cuda").manual_seed(90), device="cuda")
    x[1, 0, 7] = value
    for _ in range(2):
        qe.qe_cache_append(c, x, x, torch.tensor([slot, 5], device="cuda"))
        got = []
        while (status := qe.qe_sync_status()) != qe.QE_OK and len(got) < 5:
            got.append(status)
        assert got == want
