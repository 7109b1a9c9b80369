"""A quantized attention layer that answers: weights on QuantEase's grids, keys and values in the 4-bit cache.

    python examples/quantized_attention.py            # needs the GPU and the built libqe.so

The four projections of an attention layer are quantized from calibration inputs and stay quantized: their products are
formed from the codes.  A prompt that all sequences share goes through the layer once; then a batch of prompts behind it in
one ragged call (pages and slots for their tokens, projections, norms and rotation of queries and keys, attention), after
which every sequence is decoded token by token.  The same is computed with the unquantized layer and keys and values in
binary32, and the relative distance of the results is printed for each stage.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_01885_gb300 import inputs, qe  # noqa: E402


def quantized(W: torch.Tensor, X: torch.Tensor, bits: int, iters: int) -> dict:
    """Codes, scales and zeros that QuantEase leaves."""
    return qe.qe_quantize_layer(W, qe.qe_build_sigma(X), bits, iters)


def normed_and_rotated(x, positions, theta=10000.0):
    """Heads over their root mean square, then pair (i, i + dim / 2) turned by position theta^(-2 i / dim), in binary32."""
    x = x.float()
    x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    half = x.shape[-1] // 2
    angle = (positions.double()[:, None] * theta ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)).float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


def plain_attention(q, k, v, heads_per_kv):
    """softmax(q k^T / sqrt(d)) v in binary32, the rows at the end of the sequence."""
    k, v = k.float().repeat_interleave(heads_per_kv, 1), v.float().repeat_interleave(heads_per_kv, 1)
    s = torch.einsum("ihd,jhd->hij", q.float(), k) / q.shape[-1] ** 0.5
    n, m = s.shape[1:]
    s = s.masked_fill(torch.arange(m, device=q.device) > torch.arange(m - n, m, device=q.device)[:, None], float("-inf"))
    return torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v)


def run(width: int = 512, heads: int = 8, kv_heads: int = 2, bits: int = 4, shared: int = 320, prompts=(200, 75, 33), steps: int = 8,
        group: int = 32, seed: int = 0) -> dict:
    dev, dim, page = "cuda", width // heads, 32
    sizes = dict(q=heads * dim, k=kv_heads * dim, v=kv_heads * dim)
    X = inputs.calib_inputs(width, 4096, dtype=torch.bfloat16, seed=seed, device=dev, heavy_frac=0.02, heavy_mult=10.0)
    W = {n: inputs.layer_weights(r, width, dtype=torch.bfloat16, seed=seed + i, device=dev, std=width ** -0.5)
         for i, (n, r) in enumerate(dict(sizes, o=width).items())}
    parts = [quantized(W[n], X, bits, 10) for n in ("q", "k", "v")]
    What = {"qkv": qe.QuantizedWeights(*(torch.cat([p[x] for p in parts]) for x in ("codes", "scales", "zeros")), bits)}
    ones, rope = torch.ones(dim, dtype=torch.bfloat16, device=dev), qe.Rope(dim)

    cache = qe.KVCache(64, page, kv_heads, dim, group)
    pool = qe.PagePool(cache)
    g = torch.Generator(device=dev).manual_seed(seed)
    errors = {}

    def layer(h, table, kv_len, new, max_q, max_kv, past, prefix_pages=None, prefix=0, what="prompt"):
        """One call for the whole batch: h holds each sequence's new[b] rows, `past` what came before them."""
        start, slots, positions = qe.qe_cache_grow(cache, pool, kv_len, new, table, h.shape[0], prefix=prefix)
        qkv = qe.qe_linear(What["qkv"], h).unflatten(-1, (heads + 2 * kv_heads, dim))          # sliced below, not copied
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        qe.qe_norm_rotate(q, k, positions, rope, q_weight=ones, k_weight=ones, q_out=q, k_out=k)
        qe.qe_cache_append(cache, k, v, slots)
        if prefix:
            out = qe.qe_cache_attention_shared(cache, q, start, kv_len, table, max_q, max_kv, prefix_pages, prefix)
        else:
            out = qe.qe_cache_attention(cache, q, start, kv_len, table, max_q, max_kv)
        y = out.flatten(1)
        if "o" not in What:                        # the output projection is quantized for what attention gives
            o = quantized(W["o"], y.T.contiguous(), bits, 10)
            What["o"] = qe.QuantizedWeights(o["codes"], o["scales"], o["zeros"], bits)
        y, want, at = qe.qe_linear(What["o"], y), [], 0
        for b, n in enumerate(new.tolist()):
            past[b] = torch.cat([past[b], h[at:at + n]])
            at, j = at + n, torch.arange(past[b].shape[0], device=dev)
            q, k, v = ((x @ W[m].T).unflatten(-1, (-1, dim)) for x, m in ((past[b][-n:], "q"), (past[b], "k"), (past[b], "v")))
            want.append(plain_attention(normed_and_rotated(q, j[-n:]), normed_and_rotated(k, j), v, heads // kv_heads).flatten(1)
                        @ W["o"].float().T)
        want = torch.cat(want)
        errors[what] = max(errors.get(what, 0.0), ((y.float() - want).norm() / want.norm()).item())

    def rows(n):
        return torch.randn(n, width, generator=g, device=dev).to(torch.bfloat16)

    def integers(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    past = [rows(0)]
    first = torch.full((1, -(-shared // page)), -1, dtype=torch.int32, device=dev)
    layer(rows(shared), first, integers([0]), integers([shared]), shared, shared, past)
    past, longest = past * len(prompts), shared + max(prompts)
    table = torch.full((len(prompts), -(-(longest + steps) // page)), -1, dtype=torch.int32, device=dev)
    kv_len = integers([shared] * len(prompts))
    layer(rows(sum(prompts)), table, kv_len, integers(prompts), max(prompts), longest, past, first[0], shared)
    for i in range(steps):
        layer(rows(len(prompts)), table, kv_len, integers([1] * len(prompts)), 1, longest + 1 + i, past, first[0], shared, "step")
    status = qe.qe_sync_status()
    assert status == qe.QE_OK, qe.qe_status_string(status)
    return errors


if __name__ == "__main__":
    for bits in (3, 4, 8):
        e = run(bits=bits)
        print(f"{bits}-bit weights, 4-bit keys and values: relative distance to the unquantized layer: "
              f"prompt {e['prompt']:.3f}, single tokens {e['step']:.3f}")
