"""Positions of the norms and rotation without a GPU: what the library is given, and refusals."""
import ctypes

import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.test_serving_abi import filled
from tests.test_serving_python import integers, world  # noqa: F401


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_lib()
    return qe.load()


def heads_given(rec):
    return qe.QEHeads.from_buffer_copy(rec.calls[-1]["args"][0] + b"\0" * 8)


def test_positions_go_along_without_a_rotation(world):  # noqa: F811
    """Tokens with negative positions are passed over where only norms are asked for, too."""
    rec = world[3]
    q, weight, positions = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.ones(64), integers(3)
    qe.qe_norm_rotate(q, None, positions, None, q_weight=weight, q_out=q)
    got = heads_given(rec)
    assert got.positions == positions.data_ptr() and got.rope is None
    qe.qe_norm_rotate(q, None, None, None, q_weight=weight, q_out=q)
    assert heads_given(rec).positions is None
    for bad in (integers(2), positions.long(), integers(3, 1), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            qe.qe_norm_rotate(q, None, bad, None, q_weight=weight)


@pytest.mark.parametrize("q_given,k_given", [(False, False), (True, False), (False, True), (True, True)])
def test_results_that_are_allocated_are_cleared(world, q_given, k_given):  # noqa: F811
    rec, q, positions = world[3], torch.zeros(3, 4, 64, dtype=torch.bfloat16), integers(3)
    kw = dict(q_out=torch.empty_like(q) if q_given else None, k_out=torch.empty_like(q) if k_given else None)
    qe.qe_norm_rotate(q, q, positions, None, **kw)
    assert heads_given(rec).clear == (not q_given) + 2 * (not k_given)
    qe.qe_norm_rotate(q, q, None, None, **kw)
    assert heads_given(rec).clear == 0


def test_other_bits_are_refused(lib):
    h = filled(qe.QEHeads, dict(tokens=5, q_heads=4, head_dim=64, dtype=qe.QE_BF16, Q=0x1000, q_token=256, q_head=64, q_out=0x3000, qo_token=256, qo_head=64))
    for clear in (4, -1, 256):
        h.clear = clear
        assert lib.qe_norm_rotate(ctypes.addressof(h), None) == qe.QE_ERR_INVALID_ARG
