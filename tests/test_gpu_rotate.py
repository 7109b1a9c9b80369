"""Norms and rotation of queries and keys against binary64.

Tolerance of a result y = a cos - b sin (a, b normed, in binary32): half a unit of its type; the norm's sum of up to 256
squares, square root, division and two products, under 2^-20 of a and of b; the angle, 2^-25 of half a turn from its
conversion and two units of sin and cos, under 2^-21 of them.  So half a unit of |y| + 2^-19 (|a| + |b|)."""
import decimal
import math

import pytest
import torch

from paper_2309_01885_gb300 import build, qe

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_lib()
    return qe.load()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def plain(x, pos, inv_freq, interleaved, w, eps):
    """(y, allowed error), binary64."""
    y = x.double()
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    out, size = y.clone(), y.abs()
    if inv_freq is not None:
        n = len(inv_freq)
        f = torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
        t = (pos.double()[:, None] * f)[:, None]         # positions up to 2^20: 2^-33 of a radian
        i = torch.arange(n, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        out[..., a] = y[..., a] * t.cos() - y[..., b] * t.sin()
        out[..., b] = y[..., b] * t.cos() + y[..., a] * t.sin()
        size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, 1.01 * HALF_ULP[x.dtype] * out.abs() + 2.0 ** -19 * size + SMALLEST[x.dtype]


def check(got, x, *how):
    want, tol = plain(x, *how)
    assert got.dtype == x.dtype and got.shape == x.shape
    err = (got.double() - want).abs()
    assert (err <= tol).all(), f"{(err > tol).sum().item()} off, up to {(err / tol).max().item():.2f} of the allowed"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,rot,interleaved,norm", [
    (1, 32, 8, 128, 128, False, True), (1, 1, 1, 64, 64, True, True), (5, 12, 12, 64, 64, False, False), (7, 71, 1, 64, 32, False, True),
    (33, 32, 32, 80, 80, False, True), (3, 16, 16, 96, 48, True, True), (9, 4, 2, 128, 36, False, True), (2, 3, 5, 8, 8, False, True),
    (4, 5, 2, 256, 256, False, True), (6, 5, 2, 192, 192, True, True), (6, 3, 1, 136, 2, False, True), (700, 232, 8, 64, 64, False, True),
    (2500, 6, 2, 128, 128, False, True), (2433, 5, 3, 64, 32, True, False), (3000, 2, 1, 72, 70, False, True), (11, 4, 4, 128, 0, False, True)])
def test_against_binary64(dtype, tokens, heads, kv_heads, dim, rot, interleaved, norm):
    g = gen(tokens + dim + rot)
    fused = torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g, device="cuda").mul_(3.0).to(dtype)
    q, k = fused[:, :heads], fused[:, heads:heads + kv_heads]           # as they lie in the fused projection's output
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    wq, wk = ((1 + torch.randn(dim, generator=g, device="cuda")).to(dtype) for _ in range(2)) if norm else (None, None)
    rope = qe.Rope(rot, theta=500000.0, interleaved=interleaved) if rot else None
    freq = [500000.0 ** (-2.0 * i / rot) for i in range(rot // 2)] if rot else None
    before = fused.clone()
    qo, ko = qe.qe_norm_rotate(q, k, pos if rot else None, rope, q_weight=wq, k_weight=wk, eps=1e-5)
    assert qe.qe_sync_status() == qe.QE_OK and fused.equal(before)
    check(qo, q, pos, freq, interleaved, wq, 1e-5)
    check(ko, k, pos, freq, interleaved, wk, 1e-5)
    # in place, where they lie
    qe.qe_norm_rotate(q, k, pos if rot else None, rope, q_weight=wq, k_weight=wk, eps=1e-5, q_out=q, k_out=k)
    assert q.equal(qo) and k.equal(ko) and fused[:, heads + kv_heads:].equal(before[:, heads + kv_heads:])


@pytest.mark.parametrize("offset", [1, 2, 4, 7])
def test_any_alignment(offset):
    tokens, heads, dim = 10, 3, 64
    flat = torch.randn(tokens * (heads * 70 + 9) + 16, generator=gen(offset), device="cuda").to(torch.float16)
    q = flat.as_strided((tokens, heads, dim), (heads * 70 + 9, 70, 1), offset)
    pos, rope = torch.arange(tokens, dtype=torch.int32, device="cuda") * 1000, qe.Rope(64)
    w = torch.randn(dim + 1, device="cuda")[1:]
    out = torch.full((tokens, heads + 1, dim + 3), 7.0, dtype=torch.float16, device="cuda")
    got, none = qe.qe_norm_rotate(q, None, pos, rope, q_weight=w, q_out=out[:, :heads, 2:2 + dim])
    assert none is None and (out[:, heads:] == 7).all() and (out[..., :2] == 7).all() and (out[..., 2 + dim:] == 7).all()
    check(got, q, pos, [10000.0 ** (-2.0 * i / 64) for i in range(32)], False, w, 1e-6)


def test_far_positions_and_any_frequency():
    """Angles of far positions, against ones worked out in sixty digits.  Frequencies are held to 2^-63 of a turn: 2^31
    positions make 2^-32 of one, which is below what is allowed anyway."""
    decimal.getcontext().prec = 60
    two_pi = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    freq = [1.0, 0.5, 1e-9, 2.0 * math.pi, 100.0, -0.3, 0.0, 3.0e-4]
    at = [0, 1, 2, 1 << 20, (1 << 31) - 1]
    angle = torch.tensor([[float(p * decimal.Decimal(f) % two_pi) for f in freq] for p in at], dtype=torch.float64, device="cuda")[:, None]
    pos = torch.tensor(at, dtype=torch.int32, device="cuda")
    x = torch.randn(5, 2, 16, generator=gen(3), device="cuda")
    for a, b, interleaved in ((slice(0, 8), slice(8, 16), False), (slice(0, 16, 2), slice(1, 16, 2), True)):
        got, _ = qe.qe_norm_rotate(x, None, pos, qe.Rope(16, interleaved=interleaved, inv_freq=freq))
        p, q = x[..., a].double(), x[..., b].double()
        for part, want in ((a, p * angle.cos() - q * angle.sin()), (b, q * angle.cos() + p * angle.sin())):
            off = (got[..., part].double() - want).abs() / (2.0 ** -19 * (p.abs() + q.abs()) + 2.0 ** -24 * want.abs())
            assert off.max().item() <= 1.0


def test_negative_positions_are_left():
    pos = torch.tensor([3, -1, 5, -7], dtype=torch.int32, device="cuda")
    x = torch.randn(4, 3, 64, generator=gen(4), device="cuda")
    out = torch.full_like(x, 9.0)
    qe.qe_norm_rotate(None, x, pos, qe.Rope(64), k_out=out)
    assert (out[[1, 3]] == 9.0).all()
    check(out[[0, 2]], x[[0, 2]], pos[[0, 2]], [10000.0 ** (-2.0 * i / 64) for i in range(32)], False, None, 0.0)


def test_not_finite_stays_in_its_head():
    x = torch.randn(4, 3, 128, generator=gen(5), device="cuda").to(torch.bfloat16)
    pos, w = torch.arange(4, dtype=torch.int32, device="cuda"), torch.ones(128, device="cuda")
    clean, _ = qe.qe_norm_rotate(x, None, pos, qe.Rope(128), q_weight=w)
    y = x.clone()
    y[1, 2, 5], y[2, 0, 100] = float("nan"), float("inf")
    got, _ = qe.qe_norm_rotate(y, None, pos, qe.Rope(128), q_weight=w)
    same = torch.ones(4, 3, dtype=torch.bool, device="cuda")
    same[1, 2] = same[2, 0] = False
    assert got[same].equal(clean[same]) and got[1, 2].isnan().all() and got[2, 0].isnan().any()
    zero, _ = qe.qe_norm_rotate(torch.zeros_like(x), None, pos, qe.Rope(128), q_weight=w, eps=1e-6)
    assert (zero == 0).all()


def test_captured_and_on_another_stream():
    x = torch.randn(50, 8, 128, generator=gen(6), device="cuda").to(torch.bfloat16)
    pos, rope = torch.arange(50, dtype=torch.int32, device="cuda"), qe.Rope(128)
    want, _ = qe.qe_norm_rotate(x, None, pos, rope)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, _ = qe.qe_norm_rotate(x, None, pos, rope, stream=s)
    s.synchronize()
    assert got.equal(want)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(x)
    with torch.cuda.graph(graph):
        qe.qe_norm_rotate(x, None, pos, rope, q_out=out)
    del rope                                             # its frequencies went along with the launch
    x.copy_(torch.randn(50, 8, 128, generator=gen(7), device="cuda"))
    graph.replay()
    check(out, x, pos, [10000.0 ** (-2.0 * i / 128) for i in range(64)], False, None, 0.0)


def test_nothing_to_do():
    q, k = qe.qe_norm_rotate(torch.empty(0, 4, 64, device="cuda"), torch.empty(0, 2, 64, device="cuda"),
                             torch.empty(0, dtype=torch.int32, device="cuda"), qe.Rope(64))
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


@pytest.mark.parametrize("tokens", [608, 1215, 1216, 1300, 1900, 2440, 3100, 3700, 4300, 4863, 4864, 4870])
def test_tokens_a_block(tokens):
    """Every number of tokens that a block may take, with a last block that lacks some, and tokens that are left as they were."""
    g = gen(tokens)
    q, k = (torch.randn(tokens, n, 64, generator=g, device="cuda").to(torch.bfloat16) for n in (3, 1))
    pos = torch.randint(-3, 1 << 16, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    pos[-2:] = torch.tensor([-1, 5], dtype=torch.int32)
    w = (1 + torch.randn(64, generator=g, device="cuda")).to(torch.bfloat16)
    freq = [10000.0 ** (-2.0 * i / 64) for i in range(32)]
    out = [torch.full_like(x, 7.0) for x in (q, k)]
    qe.qe_norm_rotate(q, k, pos, qe.Rope(64), q_weight=w, k_weight=w, q_out=out[0], k_out=out[1])
    on = pos >= 0
    for x, y in zip((q, k), out):
        assert (y[~on] == 7.0).all()
        check(y[on], x[on], pos[on], freq, False, w, 1e-6)
