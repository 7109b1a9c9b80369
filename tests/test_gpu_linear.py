"""Products with a quantized layer against binary64.

Codes less zeros and x are held exactly, so a sum's error is that of adding.  With S = sum_j |s (c - z) x_j|: a chain of
accumulations on the matrix units is up to p / 16 long (sixteen columns are added at once; some 40 more for the joining), each
off by a unit of binary32, 2^-23 of what is there.  That is at most S where all terms have one sign.  Where they have either, as in
most of these tests, it is a random walk's end, below S / 8 from some 100 columns on: (p / 128 + 40) 2^-23 S.  Activations
are steeper than 1 by at most 13%, and their functions are off by a few units: 2^-20 of the result and of S's error.
Then half a unit of the result's type."""
import math

import pytest
import torch

from paper_2309_01885_gb300 import build, qe

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def layer(q, p, bits, group, seed):
    g, top = gen(seed), 2 ** bits - 1
    groups = -(-p // group) if 0 < group < p else 1
    codes = torch.randint(0, top + 1, (q, p), generator=g, device="cuda", dtype=torch.uint8)
    scales = (0.2 + torch.rand(q, groups, generator=g, device="cuda")) / (top * math.sqrt(p))
    zeros = torch.randint(0, top + 1, (q, groups), generator=g, device="cuda").float()
    if groups == 1:
        scales, zeros = scales[:, 0].contiguous(), zeros[:, 0].contiguous()
    return codes, scales, zeros


def weights64(codes, scales, zeros, group):
    q, p = codes.shape
    s, z = (v.double().view(q, -1) for v in (scales, zeros))
    if s.shape[1] > 1:
        s, z = (v.repeat_interleave(group, 1)[:, :p] for v in (s, z))
    return s * (codes.double() - z)


def plain(w, x, bias, act, residual, chain=128):
    """(y, allowed error), binary64."""
    y, size = x.double() @ w.T, x.double().abs() @ w.abs().T
    tol = size * ((x.shape[1] / chain + 40) * 2.0 ** -23)
    if bias is not None:
        y = y + bias.double()
        tol = tol + y.abs() * 2.0 ** -23
    if act == "relu":
        y = y.clamp(min=0.0)
    elif act == "silu":
        y = y * torch.sigmoid(y)
    elif act == "gelu":
        y = 0.5 * y * torch.erfc(-y / math.sqrt(2.0))
    elif act == "gelu_tanh":
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    tol = 1.15 * tol + y.abs() * 2.0 ** -20 + 2.0 ** -140
    if residual is not None:
        y = y + residual.double()
        tol = tol + y.abs() * 2.0 ** -23
    return y, tol + 1.01 * HALF_ULP[x.dtype] * y.abs() + SMALLEST[x.dtype]


def check(got, w, x, bias=None, act="none", residual=None, chain=128):
    want, tol = plain(w, x, bias, act, residual, chain)
    assert got.dtype == x.dtype and got.shape == want.shape
    over = want.abs() + tol > torch.finfo(x.dtype).max    # of these infinity is an answer too
    err = torch.where(over & (got.double() == want.sign() * math.inf), 0.0, (got.double() - want).abs())
    assert bool((err <= tol).all()), f"{(err > tol).sum().item()} off, up to {(err / tol).max().item():.2f} of the allowed, first {(err > tol).nonzero()[0].tolist()}"


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
ROWS = (1, 2, 8, 9, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 200, 256, 257, 300, 513)


@pytest.mark.parametrize("bits", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("q,p,group", [(128, 256, 0), (96, 192, 64), (200, 520, 128), (17, 72, 0), (16, 64, 64), (1, 8, 0), (300, 1000, 256),
                                       (129, 65, 64), (640, 2048, 128), (5, 333, 64)])
def test_bits_and_sizes(bits, q, p, group):
    """Every number of bits, odd sizes, groups that end inside a row, and numbers of rows on both sides of every form."""
    codes, scales, zeros = layer(q, p, bits, group, q + p + bits)
    w64 = weights64(codes, scales, zeros, group)
    w = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group)
    g = gen(bits)
    for i, rows in enumerate(ROWS):
        dtype = (torch.bfloat16, torch.float16)[(i + bits) % 2]
        x = torch.randn(rows, p, generator=g, device="cuda").to(dtype)
        check(qe.qe_linear(w, x), w64, x)
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 12, 40, 150, 300])
@pytest.mark.parametrize("act", ACTS)
def test_epilogue(dtype, rows, act):
    q, p = 208, 320
    codes, scales, zeros = layer(q, p, 4, 64, rows)
    w64, w = weights64(codes, scales, zeros, 64), qe.QuantizedWeights(codes, scales, zeros, 4, group_size=64)
    g = gen(rows)
    x = torch.randn(rows, p, generator=g, device="cuda").mul_(4.0).to(dtype)
    residual = torch.randn(rows, q, generator=g, device="cuda").to(dtype)
    for bias in (None, torch.randn(q, generator=g, device="cuda"), torch.randn(q, generator=g, device="cuda").to(dtype)):
        for res in (None, residual):
            check(qe.qe_linear(w, x, bias=bias, activation=act, residual=res), w64, x, bias, act, res)
    # onto the residual stream itself
    stream = residual.clone()
    out = qe.qe_linear(w, x, activation=act, residual=stream, out=stream)
    assert out is stream
    check(out, w64, x, None, act, residual)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(act, dtype):
    """Sums from far below 0 to far above it, taken from one row of ones: fp32 functions off by 2^-19 of their value, plus
    what one unit in the last place of the sum, its distance from 0, makes (steepness up to |y| times the value in the tails)."""
    n = 4001
    want = torch.linspace(-95.0, 95.0, n, device="cuda", dtype=torch.float64)
    want[::3] *= 0.05
    codes = torch.ones(n, 64, dtype=torch.uint8, device="cuda")
    scales = (want / 64).float()
    w = qe.QuantizedWeights(codes, scales, torch.zeros(n, device="cuda"), 4)
    for rows in (1, 40):
        x = torch.ones(rows, 64, device="cuda").to(dtype)
        got = qe.qe_linear(w, x, activation=act)[0].double()
        y = scales.double() * 64
        f = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.exp(-torch.nn.functional.softplus(-v)),
             "gelu": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2.0)),
             "gelu_tanh": lambda v: v * torch.exp(-torch.nn.functional.softplus(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))}[act]
        r = f(y)
        off = 2.0 ** -19 + 2.0 ** -22 * (y * y + 1.0) * (1.0 if act in ("gelu", "gelu_tanh", "silu") else 0.0) * (1.0 + y.abs() * (act == "gelu_tanh"))
        # below 2^-126 binary32's own exponentials end
        assert bool(((got - r).abs() <= r.abs() * (1.01 * HALF_ULP[dtype] + off) + SMALLEST[dtype] + 2.0 ** -118).all())


@pytest.mark.parametrize("rows", [1, 7, 30, 70, 260])
def test_strides_and_alignment(rows):
    """x, residual and results inside wider arrays, at any alignment; what lies around the results stays."""
    q, p = 120, 200
    codes, scales, zeros = layer(q, p, 3, 0, rows)
    w64, w = weights64(codes, scales, zeros, 0), qe.QuantizedWeights(codes, scales, zeros, 3)
    g = gen(rows)
    ws = torch.empty(qe.qe_linear_workspace(w, rows), dtype=torch.uint8, device="cuda")
    for off, ld in ((0, 208), (8, 216), (1, 208), (0, 203), (3, 209), (4, 204)):
        wide = torch.full((rows, ld + 16), float("nan"), dtype=torch.bfloat16, device="cuda").flatten()
        x = wide.as_strided((rows, p), (ld, 1), off)
        x.copy_(torch.randn(rows, p, generator=g, device="cuda"))
        res = torch.randn(rows, q + 3, generator=g, device="cuda").to(torch.bfloat16)[:, 1:1 + q]
        out = torch.full((rows, q + 7), 5.0, dtype=torch.bfloat16, device="cuda")
        for workspace in (None, ws):
            qe.qe_linear(w, x, residual=res, out=out[:, 3:3 + q], workspace=workspace)
            check(out[:, 3:3 + q], w64, x, residual=res)
            assert (out[:, :3] == 5).all() and (out[:, 3 + q:] == 5).all()


def test_codes_inside_a_wider_array():
    codes, scales, zeros = layer(50, 130, 4, 0, 1)
    wide = torch.full((50, 140), 255, dtype=torch.uint8, device="cuda")
    wide[:, 5:135] = codes + 16 * torch.randint(0, 16, codes.shape, device="cuda", dtype=torch.uint8)   # only the low bits count
    w = qe.QuantizedWeights(wide[:, 5:135], scales, zeros, 4)
    x = torch.randn(3, 130, generator=gen(2), device="cuda").to(torch.float16)
    check(qe.qe_linear(w, x), weights64(codes, scales, zeros, 0), x)


@pytest.mark.parametrize("rows", [1, 20, 90, 300])
@pytest.mark.parametrize("bits", [2, 3, 4, 8])
def test_rows_are_apart(bits, rows):
    """What is not finite in a row of x, or in a layer's grid, stays in that row, or output."""
    q, p = 144, 256
    codes, scales, zeros = layer(q, p, bits, 64, bits)
    w = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=64)
    x = torch.randn(rows, p, generator=gen(rows), device="cuda").to(torch.bfloat16)
    clean = qe.qe_linear(w, x)
    y = x.clone()
    y[rows // 2, 100] = float("inf")
    got = qe.qe_linear(w, y)
    rest = [m for m in range(rows) if m != rows // 2]
    assert got[rest].equal(clean[rest]) and not got[rows // 2].isfinite().any()
    assert qe.qe_sync_status() == qe.QE_OK
    for bad_s, bad_z in ((float("nan"), None), (float("inf"), None), (None, 2.0 ** bits), (None, -1.0), (None, 0.5), (None, float("nan"))):
        s, z = scales.clone(), zeros.clone()
        if bad_s is not None:
            s[77, 2] = bad_s
        else:
            z[77, 2] = bad_z
        got = qe.qe_linear(qe.QuantizedWeights(codes, s, z, bits, group_size=64), x)
        assert qe.qe_sync_status() == qe.QE_ERR_NUMERIC
        rest = [i for i in range(q) if i != 77]
        assert got[:, rest].equal(clean[:, rest]) and got[:, 77].isnan().all()


@pytest.mark.parametrize("rows", [1, 5, 24, 64, 500])
def test_same_answer_every_time(rows):
    codes, scales, zeros = layer(1000, 4096, 3, 128, rows)
    w = qe.QuantizedWeights(codes, scales, zeros, 3, group_size=128)
    x = torch.randn(rows, 4096, generator=gen(rows), device="cuda").to(torch.bfloat16)
    first = qe.qe_linear(w, x)
    check(first, weights64(codes, scales, zeros, 128), x)
    for _ in range(20):
        assert qe.qe_linear(w, x).equal(first)


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("q,p,rows,group", [(4096, 8320, 4000, 0), (4000, 2112, 5000, 64), (4096, 4160, 3000, 128), (2048, 20000, 300, 0), (30000, 320, 400, 0),
                                            (40000, 200, 60, 0), (40000, 200, 100, 64)])
def test_many_tiles(bits, q, p, rows, group):
    """More tiles than there are CTAs, each with many steps: rings go round hundreds of times, and answers do not change."""
    codes, scales, zeros = layer(q, p, bits, group, q + p + bits)
    w = qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group)
    x = torch.randn(rows, p, generator=gen(bits), device="cuda").to(torch.bfloat16)
    first = qe.qe_linear(w, x)
    check(first, weights64(codes, scales, zeros, group), x)
    for _ in range(5):
        assert qe.qe_linear(w, x).equal(first)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 33, 300])
def test_small_and_large_x(dtype, rows):
    """Subnormal x, and x near the end of its type, keep their bits."""
    codes, scales, zeros = layer(64, 128, 4, 0, 5)
    zeros.clamp_(max=7.0)
    codes.clamp_(min=8)                                  # differences above 0: no cancellation in what is compared
    w64, w = weights64(codes, scales, zeros, 0), qe.QuantizedWeights(codes, scales, zeros, 4)
    x = (1.0 + torch.rand(rows, 128, generator=gen(6), device="cuda"))
    tiny = (x * (2.0 ** -24 if dtype is torch.float16 else 2.0 ** -110)).to(dtype)
    check(qe.qe_linear(w, tiny), w64, tiny)
    big = (x * (2.0 ** 14 if dtype is torch.float16 else 2.0 ** 100)).to(dtype)
    check(qe.qe_linear(w, big), w64, big)


@pytest.mark.parametrize("rows", [1, 40, 400])
def test_captured_and_on_another_stream(rows):
    codes, scales, zeros = layer(256, 512, 4, 0, rows)
    w = qe.QuantizedWeights(codes, scales, zeros, 4)
    x = torch.randn(rows, 512, generator=gen(1), device="cuda").to(torch.bfloat16)
    want = qe.qe_linear(w, x, activation="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = qe.qe_linear(w, x, activation="silu", stream=s)
    s.synchronize()
    assert got.equal(want)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        qe.qe_linear(w, x, activation="silu", out=out)
        qe.qe_linear(w, x, activation="silu", residual=out, out=out)
    y = torch.randn(rows, 512, generator=gen(2), device="cuda").to(torch.bfloat16)
    x.copy_(y)
    graph.replay()
    one = qe.qe_linear(w, y, activation="silu")
    assert out.equal(qe.qe_linear(w, y, activation="silu", residual=one))


def test_a_quantized_layer_as_it_comes():
    """qe_quantize_layer's own codes and grids, grouped and not, multiply as the weights that they stand for."""
    from paper_2309_01885_gb300 import inputs
    W = inputs.layer_weights(256, 512, dtype=torch.bfloat16, device="cuda")
    X = inputs.calib_inputs(512, 2048, dtype=torch.bfloat16, device="cuda")
    Sigma = qe.qe_build_sigma(X)
    for bits, group in ((3, 0), (4, 256), (8, 0)):
        out = qe.qe_quantize_layer(W, Sigma, bits, 3, group_size=group)
        w = qe.QuantizedWeights(out["codes"], out["scales"], out["zeros"], bits, group_size=group)
        w64 = weights64(out["codes"], out["scales"], out["zeros"], group)
        for rows in (2, 50, 700):
            x = X[:, :rows].T.contiguous()
            check(qe.qe_linear(w, x), w64, x)
    assert qe.qe_sync_status() == qe.QE_OK


def test_no_rows():
    codes, scales, zeros = layer(64, 128, 4, 0, 5)
    w = qe.QuantizedWeights(codes, scales, zeros, 4)
    assert qe.qe_linear(w, torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")).shape == (0, 64)


@pytest.mark.parametrize("rows,q,p,group", [(70000, 40, 128, 0), (3, 200000, 64, 0), (300, 150000, 64, 0), (2, 16, 1 << 20, 0), (50, 33, 1 << 18, 0),
                                            (2, 16, 1 << 18, 64), (100, 130, 1 << 16, 128)])
@pytest.mark.parametrize("bits", [3, 4])
def test_long_axes(rows, q, p, group, bits):
    codes, scales, zeros = layer(q, p, bits, group, bits)
    x = torch.randn(rows, p, generator=gen(6), device="cuda").to(torch.bfloat16)
    got = qe.qe_linear(qe.QuantizedWeights(codes, scales, zeros, bits, group_size=group), x)
    w = weights64(codes, scales, zeros, group)
    for i in range(0, rows, 10000):
        check(got[i:i + 10000], w, x[i:i + 10000])
    assert qe.qe_sync_status() == qe.QE_OK


@pytest.mark.parametrize("rows", [1, 20, 64, 300])
@pytest.mark.parametrize("p,group", [(1000, 0), (40000, 0), (40000, 128)])
def test_terms_of_one_sign(rows, p, group):
    codes, scales, zeros = layer(48, p, 4, group, p)
    zeros.zero_()
    x = torch.rand(rows, p, generator=gen(7), device="cuda").to(torch.float16)
    check(qe.qe_linear(qe.QuantizedWeights(codes, scales, zeros, 4, group_size=group), x), weights64(codes, scales, zeros, group), x, chain=16)
