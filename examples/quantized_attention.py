"""A quantized attention layer that answers: weights on QuantEase's grids, keys and values in the 4-bit cache.

    python examples/quantized_attention.py            # needs the GPU and the built libqe.so

The four projections of an attention layer are quantized from calibration inputs.  A batch of prompts
then goes through the layer in one ragged call (append its keys and values, attend over them), after which
every sequence is decoded token by token.  The same is computed with the unquantized layer and keys and
values in binary32, and the relative distance of the results is printed for each stage.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_01885_gb300 import inputs, qe  # noqa: E402


class PagedSequences:
    """Pages handed out to sequences as they grow: the page table and the slots of new tokens."""

    def __init__(self, cache: qe.KVCache, seqs: int, max_len: int):
        self.page = cache.page_size
        self.table = torch.full((seqs, -(-max_len // self.page)), -1, dtype=torch.int32)
        self.length = [0] * seqs
        self.free = list(range(cache.pages))
        self.device = cache.device

    def grow(self, seq: int, tokens: int) -> torch.Tensor:
        """Slots of the next `tokens` tokens of sequence `seq`."""
        j = torch.arange(self.length[seq], self.length[seq] + tokens)
        for p in range(-(-self.length[seq] // self.page), -(-(self.length[seq] + tokens) // self.page)):
            self.table[seq, p] = self.free.pop()
        self.length[seq] += tokens
        return self.table[seq, j // self.page].long() * self.page + j % self.page

    def lengths(self) -> torch.Tensor:
        return torch.tensor(self.length, dtype=torch.int32, device=self.device)


def quantized_projection(W: torch.Tensor, X: torch.Tensor, bits: int, iters: int) -> torch.Tensor:
    """The weights that QuantEase leaves, in bf16."""
    out = qe.qe_quantize_layer(W, qe.qe_build_sigma(X), bits, iters)
    return (out["scales"][:, None] * (out["codes"].float() - out["zeros"][:, None])).to(torch.bfloat16)


def plain_attention(q, k, v, heads_per_kv):
    """softmax(q k^T / sqrt(d)) v in binary32, the rows at the end of the sequence."""
    k, v = k.float().repeat_interleave(heads_per_kv, 1), v.float().repeat_interleave(heads_per_kv, 1)
    s = torch.einsum("ihd,jhd->hij", q.float(), k) / q.shape[-1] ** 0.5
    n, m = s.shape[1:]
    s = s.masked_fill(torch.arange(m, device=q.device) > torch.arange(m - n, m, device=q.device)[:, None], float("-inf"))
    return torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v)


def run(width: int = 512, heads: int = 8, kv_heads: int = 2, bits: int = 4, prompts=(200, 75, 33), steps: int = 8,
        group: int = 32, seed: int = 0) -> dict:
    dev, dim = "cuda", width // heads
    sizes = dict(q=heads * dim, k=kv_heads * dim, v=kv_heads * dim)
    X = inputs.calib_inputs(width, 4096, dtype=torch.bfloat16, seed=seed, device=dev, heavy_frac=0.02, heavy_mult=10.0)
    W = {n: inputs.layer_weights(r, width, dtype=torch.bfloat16, seed=seed + i, device=dev, std=width ** -0.5)
         for i, (n, r) in enumerate(dict(sizes, o=width).items())}
    What = {n: quantized_projection(w, X, bits, 10) for n, w in W.items() if n != "o"}
    fused = torch.cat([What["q"], What["k"], What["v"]])

    cache = qe.KVCache(64, 32, kv_heads, dim, group)
    paged = PagedSequences(cache, len(prompts), max(prompts) + steps)
    g = torch.Generator(device=dev).manual_seed(seed)
    kept = [[] for _ in prompts]                   # the hidden states so far, for the unquantized layer
    errors = {}

    def layer(hidden: list, what: str):
        """One call for the whole batch: `hidden` holds each sequence's new rows."""
        rows = [h.shape[0] for h in hidden]
        h = torch.cat(hidden)
        qkv = (h @ fused.T).unflatten(-1, (heads + 2 * kv_heads, dim))     # sliced below, not copied
        slots = torch.cat([paged.grow(b, n) for b, n in enumerate(rows)]).to(dev)
        qe.qe_cache_append(cache, qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], slots)
        start = torch.tensor([0] + rows, device=dev).cumsum(0).to(torch.int32)
        out = qe.qe_cache_attention(cache, qkv[:, :heads], start, paged.lengths(), paged.table.to(dev), max(rows), max(paged.length))
        y = out.flatten(1)
        if what == "prompt":                       # the output projection sees what attention gives
            What["o"] = quantized_projection(W["o"], y.T.contiguous(), bits, 10)
        y = y @ What["o"].T
        want = []
        for b, n in enumerate(rows):
            kept[b].append(hidden[b])
            past = torch.cat(kept[b])
            q, k, v = ((x @ W[m].T).unflatten(-1, (-1, dim)) for x, m in ((hidden[b], "q"), (past, "k"), (past, "v")))
            want.append(plain_attention(q, k, v, heads // kv_heads).flatten(1) @ W["o"].float().T)
        want = torch.cat(want)
        errors[what] = max(errors.get(what, 0.0), ((y.float() - want).norm() / want.norm()).item())
        return y

    layer([torch.randn(n, width, generator=g, device=dev).to(torch.bfloat16) for n in prompts], "prompt")
    for _ in range(steps):
        layer([torch.randn(1, width, generator=g, device=dev).to(torch.bfloat16) for _ in prompts], "step")
    status = qe.qe_sync_status()
    assert status == qe.QE_OK, qe.qe_status_string(status)
    return errors


if __name__ == "__main__":
    for bits in (3, 4, 8):
        e = run(bits=bits)
        print(f"{bits}-bit weights, 4-bit keys and values: relative distance to the unquantized layer: "
              f"prompt {e['prompt']:.3f}, single tokens {e['step']:.3f}")
