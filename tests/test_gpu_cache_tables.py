"""Attention over the 4-bit cache with page tables that are parts of others."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.test_gpu_cache import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("q_len", [1, 40])
def test_parts_of_a_wider_table(q_len):
    b = Batch([q_len, q_len], [200, 90], 4, 2, 64, 32, 16, torch.bfloat16, seed=70)
    want = b.run()
    table, seqs, width = b.table, *b.table.shape
    wide = torch.full((2 * seqs, width + 7), 1 << 20, dtype=torch.int32, device="cuda")   # pages that the cache does not have
    wide[::2, 3:3 + width] = table
    b.table = wide[::2, 3:3 + width]
    assert torch.equal(b.run(), want)
    b.table = table.t().contiguous().t()
    assert torch.equal(b.run(), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = b.run(stream=s)
    s.synchronize()
    assert torch.equal(out, want) and qe.qe_sync_status() == qe.QE_OK
    # tokens past the part's own columns are reported and not there, whatever stands beside it
    b.table = wide[::2, 3:3 + width - 1]
    b.kv_lens[0] = b.table.shape[1] * 16 + 1
    b.run()
    assert qe.qe_sync_status() == qe.QE_ERR_INVALID_ARG


def test_a_row_that_was_a_column():
    b = Batch([1], [150], 4, 2, 64, 32, 16, torch.bfloat16, seed=71)
    want = b.run()
    b.table = b.table.reshape(-1, 1).t()
    assert b.table.stride() == (1, 1)
    assert torch.equal(b.run(), want) and qe.qe_sync_status() == qe.QE_OK
