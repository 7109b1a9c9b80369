"""Products with a quantized layer where their forms meet their limits (bounds: tests/test_gpu_linear.py)."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.test_gpu_linear import check, gen, layer, weights64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("rows,q,p", [(200, 4096, 4096), (256, 4096, 4096), (150, 4096, 11008)])
def test_halves_of_a_shared_tile(rows, q, p, group, bits):
    """A cluster shares a tile whose halves of rows take turns, and the last two units lie where the sums begin: the first half's
    sums have to wait for the second half's products, which still read x."""
    codes, scales, zeros = layer(q, p, bits, group, rows + p + bits)
    w = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group)
    x = torch.randn(rows, p, generator=gen(rows), device="cuda").to(torch.bfloat16)
    first = qe.qe_linear(w, x)
    check(first, weights64(codes, scales, zeros, group), x)
    for _ in range(30):
        assert qe.qe_linear(w, x).equal(first)
    assert qe.qe_sync_status() == qe.QE_OK
