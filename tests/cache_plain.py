"""Attention over the 4-bit cache in binary64, with the error that the kernels' roundings may cause.

Of each query row, with p the softmax and v the cached values (both as the cache holds them):

  scores        the keys may be rounded once to 11 bits: a score moves by at most e_j = 2^-11 scale sum |q k_j|, its
                probability by a factor within exp(e_j), and the sum of all of them by the p-weighted mean of those;
  probability   rounded to 11 bits, then its product with a value scale, or the value itself, rounded to 11 bits:
                2^-10 of each term;
  binary32      sums and exponentials: 2^-16 of each term leaves room for sequences up to 2^20 tokens;
  result        half an ulp of its type, or of its subnormals.

Every bound is relative to the terms of the same channel: no other channel's, row's or token's size enters."""
import math

import torch

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def plain(q, kv, q_len, causal=True, window=0, scale=0.0):
    """(out, lse, allowed error of out, allowed error of lse): q rows x heads x dim, kv a (keys, values) pair of
    binary64 tensors (tokens x kv heads x dim) for each sequence, q_len the rows of each."""
    dev, (rows, heads, dim) = q.device, q.shape
    scale = scale or 1.0 / math.sqrt(dim)
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device=dev)
    tol, ltol, at = torch.zeros_like(out), torch.zeros_like(lse), 0
    for n, (k, v) in zip(q_len, kv):
        m = k.shape[0]
        if n and m:
            rep = heads // k.shape[1]
            pos, j = torch.arange(m - n, m, device=dev)[:, None], torch.arange(m, device=dev)
            sees = torch.ones(n, m, dtype=torch.bool, device=dev)
            if causal:
                sees = j <= pos
                if window:
                    sees &= j > pos - window
            some = sees.any(-1)
            for h in range(heads):
                x, kk, vv = q[at:at + n, h].double(), k[:, h // rep], v[:, h // rep]
                s = (x @ kk.T * scale).masked_fill(~sees, -math.inf)
                p = torch.softmax(s, -1).masked_fill(~some[:, None], 0.0)
                moved = torch.expm1(x.abs() @ kk.abs().T * scale * 2.0 ** -11).clamp(max=1e6)
                o = p @ vv
                out[at:at + n, h] = o
                all_of = (p * moved).sum(-1)
                lse[at:at + n, h] = torch.logsumexp(s, -1)
                ltol[at:at + n, h] = 1.1 * all_of + 1e-5
                tol[at:at + n, h] = 1.1 * ((p * (moved + 2.0 ** -10 + 2.0 ** -16)) @ vv.abs() + o.abs() * all_of[:, None])
        at += n
    tol += HALF_ULP[q.dtype] * out.abs() * 1.02 + SMALLEST[q.dtype]
    return out, lse, tol, ltol


def compare(got, lse, q, kv, q_len, **how):
    """Asserts that a result (and its log sums) agree with the plain form."""
    out, want_lse, tol, ltol = plain(q, kv, q_len, **how)
    assert got.dtype == q.dtype and got.isfinite().all(), f"{(~got.isfinite()).sum().item()} results are not finite"
    err = (got.double() - out).abs()
    bad = err > tol
    assert not bad.any(), (f"{bad.sum().item()} of {bad.numel()} off, up to {(err / tol).max().item():.2f} of the allowed, "
                           f"first at {bad.nonzero()[0].tolist()}")
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (got[empty] == 0).all()
    assert ((lse.double() - want_lse)[~empty].abs() <= ltol[~empty]).all()
