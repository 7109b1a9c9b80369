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


# ---- sums of one sign ----

# Products are exact.  The matrix units add sixteen columns at a time, each addition off by a unit of binary32 at most, 2^-23 of
# what is there, and hand their sums on every 8192 columns (where a CTA of the few-rows form has up to 16384, at their end), or
# every group: 512 (1024) units of S = sum_j |s (c - z) x_j| at most, or group / 16.  These sums are added up in binary32, half a
# unit each, a CTA's share and then eight CTAs'; scales and the bias come in with half a unit each: 40 for all but the first.  The
# bias takes the sum away again, so that the result's own rounding counts for nothing.
def one_sign_units(p, group, rows):
    chain = min(p, 16384 if not group and rows <= 32 and p <= 8 * 16384 else 8192, group or p)
    return chain / 16 + p / chain / 2 + 40


def check_one_sign(rows, q, p, group, bits, dtype):
    codes, scales, zeros = layer(q, p, bits, group, p + rows)
    zeros.zero_()
    x = torch.rand(1, p, generator=gen(rows), device="cuda").to(dtype)
    w64 = weights64(codes, scales, zeros, group)
    sums = (w64 @ x[0].double())
    del w64
    bias = -sums.float()
    w = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group)
    got = qe.qe_linear(w, x.expand(rows, p).contiguous(), bias=bias).double()
    off = (got - (sums + bias.double())).abs() * 2.0 ** 23 / sums
    most = one_sign_units(p, group, rows) * (1.0 + 2.0 ** -8) + (2.0 ** -25 * 2.0 ** 23 / sums.min().item())
    assert off.max().item() <= most, f"{off.max().item():.0f} units of the sum off, of {most:.0f} allowed"
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 12, 20, 32])
@pytest.mark.parametrize("p,group,bits", [(8192, 0, 4), (1 << 17, 0, 4), (1 << 18, 0, 4), (1 << 20, 0, 4), (1 << 20, 0, 3), (1 << 20, 0, 8), ((3 << 18) + 200, 0, 4), (1 << 22, 0, 4),
                                          (1 << 20, 1 << 13, 4), (1 << 20, 1 << 17, 4), (1 << 20, 1 << 19, 3), (600000, 65600, 4)])
def test_sums_of_one_sign_few_rows(p, group, bits, rows, dtype):
    check_one_sign(rows, 40, p, group, bits, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [33, 64, 120, 300])
@pytest.mark.parametrize("p,group,bits", [(8192, 0, 4), (1 << 18, 0, 4), (1 << 20, 0, 8), (1 << 20, 1 << 13, 4), (1 << 20, 1 << 17, 4), (1 << 20, 1 << 19, 3), (600000, 65600, 4),
                                          (600000, 10048, 8)])
def test_sums_of_one_sign_many_rows(p, group, bits, rows, dtype):
    check_one_sign(rows, 40, p, group, bits, dtype)


# ---- long axes with exact sums: a column, a unit, a stage or a CTA's share that is missing or counted twice shows ----

def borders(p):
    """Columns on either side of units (64), stages (256 and 128), segments (8192) and CTAs' shares of two to eight."""
    units, at = -(-p // 64), {0, 1, p - 2, p - 1, p // 2}
    for step in (64, 128, 256, 8192, 16384):
        at |= {step - 1, step, p // step * step - 1, p // step * step, p // (2 * step) * step}
    for ranks in range(2, 9):
        for r in range(1, ranks):
            at |= {units * r // ranks * 64 - 1, units * r // ranks * 64}
    return sorted(j for j in at if 0 <= j < p)


AXES = [(130, 64, 0), (130, 1000, 0), (48, 40000, 0), (40, 100000, 0), (16, 1 << 18, 0), (16, (1 << 20) + 72, 0), (40, 40000, 128), (40, 40000, 64), (40, 200000, 16384),
        (2000, 4096, 64), (2000, 4096, 0)]


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("rows", [1, 7, 13, 20, 32, 33, 64, 100, 200])
@pytest.mark.parametrize("q,p,group", AXES)
def test_every_column_once(q, p, group, rows, bits):
    """Differences of one everywhere and x of ones: p, to the last one, which the bias takes away."""
    codes, scales, zeros = layer(q, p, bits, group, bits)
    groups = 1 if zeros.dim() == 1 else zeros.shape[1]
    zeros.clamp_(max=2.0 ** bits - 2.0)
    z = zeros.view(q, groups)
    codes = (z.repeat_interleave(group, 1)[:, :p] if groups > 1 else z.expand(q, p)).to(torch.uint8) + 1
    w = qe.QuantizedWeights(codes, torch.ones_like(scales), zeros, bits, group_size=group)
    bias = torch.full((q,), -float(p), device="cuda")
    x = torch.ones(rows, p, dtype=(torch.bfloat16, torch.float16)[bits % 2], device="cuda")
    assert (qe.qe_linear(w, x, bias=bias) == 0).all()
    x[:, p // 3] = 2.0                                    # and one of them twice
    assert (qe.qe_linear(w, x, bias=bias) == 1).all()
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("rows", [1, 8, 32, 33, 64, 200])
@pytest.mark.parametrize("q,p,group", AXES)
def test_every_column_in_its_place(q, p, group, rows, bits):
    """Rows of x with a single 1, at every border: the column itself comes out, s (c - z) rounded once."""
    codes, scales, zeros = layer(q, p, bits, group, p + bits)
    w, w64 = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group), weights64(codes, scales, zeros, group)
    at = torch.tensor(borders(p), device="cuda")
    dtype = (torch.bfloat16, torch.float16)[bits % 2]
    for lo in range(0, len(at), rows):
        cols = at[lo:lo + rows]
        x = torch.zeros(rows, p, dtype=dtype, device="cuda")
        x[torch.arange(len(cols), device="cuda"), cols] = 1.0
        got = qe.qe_linear(w, x)
        # the product of a scale and a whole number is rounded to binary32, then to the result's type
        assert got[:len(cols)].equal(w64[:, cols].T.float().to(dtype)) and (got[len(cols):] == 0).all()
    assert qe.qe_sync_status() == qe.QE_OK
