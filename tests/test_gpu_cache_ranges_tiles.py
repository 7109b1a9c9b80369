"""The value ranges of test_gpu_cache_ranges.py where there are many query rows to a kv head."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests import test_gpu_cache_ranges as ranges

pytestmark = pytest.mark.gpu

# (query heads, kv heads, dim, group), query rows: more than 32 (row, head) pairs of a kv head
MANY = [((8, 2, 128, 32), 130), ((8, 8, 128, 64), 130), ((4, 1, 64, 32), 100), ((3, 3, 96, 32), 270), ((16, 1, 128, 128), 3),
        ((40, 1, 64, 64), 1)]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("shape,q_len", MANY)
@pytest.mark.parametrize("bits", [10, 14, 20, 26])
def test_large_values_without_weight(shape, q_len, bits):
    ranges.large_values_without_weight(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", MANY)
@pytest.mark.parametrize("bits", [10, 14, 20, 26])
def test_large_values_that_are_masked(shape, q_len, bits):
    ranges.large_values_that_are_masked(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", MANY)
@pytest.mark.parametrize("bits", [8, 14, 20])
def test_channel_groups_of_different_sizes(shape, q_len, bits):
    ranges.groups_of_different_sizes(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", MANY)
@pytest.mark.parametrize("heavy,small", [(12.0, 0), (14.0, 16), (30.0, 30)])
def test_a_heavy_token_and_a_flat_tail(shape, q_len, heavy, small):
    ranges.heavy_token_and_flat_tail(shape, q_len, heavy, small)


@pytest.mark.parametrize("shape,q_len", MANY)
def test_every_token_has_its_own_size(shape, q_len):
    ranges.every_token_its_own_size(shape, q_len)
