"""Attention over the 4-bit cache where value sizes differ: between tokens whatever their weight, between the channel
groups of a head, and between a few heavy tokens and a long flat tail.  Each result is held to the size of its own
channel's terms."""
import pytest
import torch

from paper_2309_01885_gb300 import build, qe
from tests.cache_plain import compare
from tests.test_gpu_cache import Batch, gen

pytestmark = pytest.mark.gpu

# (query heads, kv heads, dim, group), query rows: up to 24 (row, head) pairs of a kv head, 32 at 64 channels
FEW = [((8, 2, 128, 32), 1), ((8, 2, 128, 32), 4), ((8, 8, 128, 64), 1), ((8, 8, 128, 64), 12), ((4, 1, 64, 32), 1), ((4, 1, 64, 32), 8),
       ((3, 3, 96, 32), 1), ((3, 3, 96, 32), 3), ((16, 1, 128, 128), 1), ((29, 1, 64, 64), 1)]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def batch(shape, q_len, n, dtype, seed):
    heads, kv_heads, dim, group = shape
    return Batch([q_len, 1], [n, 77], heads, kv_heads, dim, group, 32, dtype, seed=seed, spread=0.5)


def check(b, k, v, **how):
    """The first sequence's tokens replaced by k and v, then compared."""
    slots = b.slots(0, torch.arange(k.shape[0], device="cuda"))
    qe.qe_cache_append(b.cache, k, v, slots)
    b.kv[0] = tuple(x.double() for x in qe.qe_cache_read(b.cache, slots, torch.float32))
    lse = torch.full(b.q.shape[:2], 7.0, device="cuda")
    got = b.run(lse=lse, **how)
    assert qe.qe_sync_status() == qe.QE_OK
    compare(got, lse, b.q, b.kv, b.q_len, **how)


def tokens(b, n, seed):
    g = gen(seed)
    H, dim = b.cache.kv_heads, b.dim
    return (torch.randn(n, H, dim, generator=g, device="cuda") * 0.5, torch.randn(n, H, dim, generator=g, device="cuda") + 0.5)


def large_values_without_weight(shape, q_len, bits):
    """Tokens with values 2^bits times the others' that no row gives weight: the others' values keep their bits."""
    for dtype in (torch.bfloat16, torch.float16):
        b = batch(shape, q_len, 700, dtype, 50)
        k, v = tokens(b, 700, 51)
        far = torch.tensor([3, 40, 41, 333, 560], device="cuda")
        # the first channel alone tells far tokens apart: score -60 in natural units for every row
        b.q[..., 0] = 8.0
        k[..., 0] = 0.0
        k[far] = 0.0
        k[far, :, 0] = -60.0 / 8.0 * b.dim ** 0.5
        v[far] *= 2.0 ** bits
        check(b, k, v)
        check(b, k, v, window=200)
        # one channel group of these tokens alone
        v[far, :, :b.cache.group_size] *= 2.0 ** -bits
        check(b, k, v)


def large_values_that_are_masked(shape, q_len, bits):
    """The last token's values are 2^bits times the others': rows before it do not see it."""
    b = batch(shape, q_len, 500, torch.bfloat16, 52)
    k, v = tokens(b, 500, 53)
    v[-1] *= 2.0 ** bits
    check(b, k, v)
    v[:-1] *= 2.0 ** -bits
    check(b, k, v)


def groups_of_different_sizes(shape, q_len, bits):
    """One channel group is 2^bits smaller than the rest, in all tokens or in some."""
    b = batch(shape, q_len, 600, torch.bfloat16, 54)
    G = b.cache.group_size
    for group in range(min(2, b.dim // G)):
        k, v = tokens(b, 600, 55)
        v[..., group * G:(group + 1) * G] *= 2.0 ** -bits
        check(b, k, v)
        k, v = tokens(b, 600, 56)
        v[::2, :, group * G:(group + 1) * G] *= 2.0 ** -bits
        check(b, k, v)


def heavy_token_and_flat_tail(shape, q_len, heavy, small):
    """The first token takes nearly all of the weight (e^heavy times another's) with values 2^-small times the others'."""
    b = batch(shape, q_len, 3000, torch.bfloat16, 57)
    k, v = tokens(b, 3000, 58)
    b.q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[0] = 0.0
    k[0, :, 0] = heavy / 8.0 * b.dim ** 0.5
    v[0] *= 2.0 ** -small
    check(b, k, v)


def every_token_its_own_size(shape, q_len):
    """Value sizes spread over 2^40, in no order, all tokens of about equal weight; near the ends of binary32 too."""
    b = batch(shape, q_len, 400, torch.bfloat16, 59)
    k, v = tokens(b, 400, 60)
    f = torch.exp2(torch.randint(-20, 21, (400,), generator=gen(61), device="cuda").float())
    for size in (1.0, 2.0 ** -70, 2.0 ** 70):
        check(b, k, v * f[:, None, None] * size)


@pytest.mark.parametrize("shape,q_len", FEW)
@pytest.mark.parametrize("bits", [10, 14, 20, 26])
def test_large_values_without_weight(shape, q_len, bits):
    large_values_without_weight(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", FEW)
@pytest.mark.parametrize("bits", [10, 14, 20, 26])
def test_large_values_that_are_masked(shape, q_len, bits):
    large_values_that_are_masked(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", FEW)
@pytest.mark.parametrize("bits", [8, 14, 20, 26])
def test_channel_groups_of_different_sizes(shape, q_len, bits):
    groups_of_different_sizes(shape, q_len, bits)


@pytest.mark.parametrize("shape,q_len", FEW)
@pytest.mark.parametrize("heavy,small", [(12.0, 0), (14.0, 16), (30.0, 30)])
def test_a_heavy_token_and_a_flat_tail(shape, q_len, heavy, small):
    heavy_token_and_flat_tail(shape, q_len, heavy, small)


@pytest.mark.parametrize("shape,q_len", FEW)
def test_every_token_has_its_own_size(shape, q_len):
    every_token_its_own_size(shape, q_len)
