"""Positions of the norms and rotation without a GPU: what the library is given, and refusals."""
import pytest
import torch

from paper_2309_01885_gb300 import qe
from tests.test_serving_python import integers, world  # noqa: F401


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
