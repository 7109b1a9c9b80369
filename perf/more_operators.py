"""A serving step over quantized weights and the 4-bit key/value cache, measured: four operators.

grow    pages, slots and positions for the tokens that a batch of sequences appends.  Pages have P tokens, free pages lie in a
        ring (first, count).  Sequence b holds len_b tokens; where ends_b it gives the pages behind the shared prefix back (to the
        ring's end) and holds l0 = prefix tokens again, else l0 = len_b.  It then takes n_b tokens: pages
        ceil(l0 / P) .. ceil((l0 + n_b) / P) - 1 of its row of the page table come from the ring's front, sequences in order; token
        at position t goes to slot page_table[b][t / P] P + t mod P.  Tokens of all sequences follow one another; entries behind
        the last one are -1 (slots) and 0 (positions).
rotate  for every token and head of queries and keys: x <- x w / sqrt(mean(x^2) + eps), then each pair (a, b) of the first R
        channels by the angle position * theta^(-2 i / R): (a cos - b sin, b cos + a sin).  Pair i is channels i and i + R / 2, or
        2 i and 2 i + 1 (interleaved).
linear  y = act(x W^T + bias) + residual with weights on grids, W_ij = s_ig (c_ij - z_ig): codes c of 2 .. 8 bits, a grid (s, z)
        for each row, or for each row and group of columns.
shared  attention over the 4-bit cache for sequences whose first `prefix` tokens are the same pages: query row i of a sequence
        with n rows and L tokens (prefix, own tokens, its rows' among these) sits at t = L - n + i and sees tokens j <= t:
            out_i = sum_j softmax_j(q_i . k^_j / sqrt(head_dim)) v^_j         (a row that sees no token is zero)

The cache holds x^ = s (c - z), 4-bit codes, one grid for each token, head and group of channels: with lo = min(x, 0), hi = max(x, 0)
over a group, s = bf16((hi - lo) / 15) (at least 2^-126), z = round(-lo / s), c = clamp(round(x / s) + z, 0, 15).
Its bytes: a block for each page and head with key codes, value codes, key grids, value grids.  Channels are padded to
D = 64, 96 or 128.  Codes come in 32-bit words, tokens in blocks of 8, and word (8-token block, lane 0 .. 31, chunk w of 32
channels) stands at block * D + lane * D / 32 + w:
    keys:   lane = 4 token + t; channel 32 w + 8 t + 2 p + h at bit 4 p + 16 h (p 0 .. 3, h 0 .. 1);
    values: lane = 4 r + t; channel 32 w + 4 r + i of token 2 t + h at bit 4 i + 16 h (i 0 .. 3, h 0 .. 1).
Grids are words [token][group]: the scale's bf16 bits above z's bf16 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
# (query heads, kv heads, head dim): the attention of the LLaMA-7B (32 x 128), Falcon-180B (232 over 8 x 64) and
# OPT-125m (12 x 64) shapes that this repository quantizes, grouped and multi-query layouts, and the odd dims 80 and 96
LAYOUTS = ((32, 32, 128), (232, 8, 64), (12, 12, 64), (32, 8, 128), (71, 1, 64), (32, 32, 80), (16, 16, 96))
# layers (outputs, inputs) that this repository quantizes
LAYERS = ((768, 768), (4096, 4096), (11008, 4096), (4096, 11008), (15360, 14848), (14848, 59392))
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # one decode step of 64 sequences, four of which have come to their end
        dict(name="grow 64 x 1", op="grow", seqs=64, new_lo=1, new_hi=1, kv_lo=0, kv_hi=8000, page=64, ends=4, prefix=0),
        # prompts of ragged lengths join a large running batch that shares a prefix, in one ragged step
        dict(name="grow 1500 x 0..200", op="grow", seqs=1500, new_lo=0, new_hi=200, kv_lo=0, kv_hi=3000, page=16, ends=70, prefix=512),
        # one token: latency
        dict(name="rotate 1 token", op="rotate", tokens=1, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, far=8000, dtype="bf16"),
        # a chunk in Falcon-180B's head layout, half of the channels rotated, pairs next to each other
        dict(name="rotate 777 tokens fp16", op="rotate", tokens=777, heads=232, kv_heads=8, dim=64, rot=32, interleaved=True, norm=True, far=40000, dtype="fp16"),
        # long prompts in LLaMA-7B's head layout, positions up to a million
        dict(name="rotate 16384 tokens", op="rotate", tokens=16384, heads=32, kv_heads=32, dim=128, rot=128, interleaved=False, norm=True, far=1000000, dtype="bf16"),
        # a single token through LLaMA-7B's projection at 3 bits, added to the residual stream
        dict(name="linear 1 x 4096 x 4096", op="linear", rows=1, q=4096, p=4096, bits=3, group=0, act="none", bias=False, residual=True, dtype="bf16"),
        # a decode batch through the MLP's first layer, 4 bits in groups, its activation on the way out
        dict(name="linear 24 x 11008 x 4096", op="linear", rows=24, q=11008, p=4096, bits=4, group=128, act="silu", bias=False, residual=False, dtype="bf16"),
        # a few drafted tokens through Falcon-180B's down projection at 3 bits
        dict(name="linear 5 x 14848 x 59392", op="linear", rows=5, q=14848, p=59392, bits=3, group=0, act="none", bias=False, residual=True, dtype="fp16"),
        # prompts of 4095 tokens in all through LLaMA-7B's down projection, back into the residual stream
        dict(name="linear 4095 x 4096 x 11008", op="linear", rows=4095, q=4096, p=11008, bits=4, group=0, act="gelu", bias=True, residual=True, dtype="bf16"),
        # a decode step of a batch behind one system prompt, answers of ragged lengths, two idle places in the batch
        dict(name="shared 64 x 8K + 1K", op="shared", seqs=64, idle=2, q_lo=1, q_hi=1, prefix=8192, own_lo=1, own_hi=1000, heads=32, kv_heads=8, dim=128, group=32, page=64, dtype="bf16"),
        # the same with a short prefix that ends inside a page, where latency counts
        dict(name="shared 8 x 500 + 100", op="shared", seqs=8, idle=0, q_lo=1, q_hi=1, prefix=500, own_lo=2, own_hi=100, heads=32, kv_heads=32, dim=128, group=64, page=16, dtype="bf16"),
        # questions of 40 to 100 tokens about one long document, Falcon-180B's heads
        dict(name="shared 6 x 12000 + 100 fp16", op="shared", seqs=6, idle=0, q_lo=40, q_hi=100, prefix=12000, own_lo=40, own_hi=100, heads=232, kv_heads=8, dim=64, group=64, page=128, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {c["op"]: 0 for c in listed()}
    for c in listed():
        most[c["op"]] = max(most[c["op"]], _cost(c))
    while True:
        op = rng.choice(("grow", "rotate", "linear", "linear", "shared", "shared"))
        dtype = rng.choice(("bf16", "fp16"))
        if op == "grow":
            seqs, page, kv = _log(rng, 1, 1500), rng.choice((16, 32, 64, 128, 256)), _log(rng, 16, 16384)
            hi = rng.choice((1, 1, _log(rng, 2, 16), _log(rng, 16, 4096)))
            c = dict(op=op, seqs=seqs, new_lo=rng.choice((0, hi // 2, hi)), new_hi=hi, kv_lo=rng.randint(0, kv), kv_hi=kv, page=page,
                     ends=rng.randint(0, seqs // 4), prefix=page * rng.choice((0, 0, rng.randint(0, kv // page))))
        elif op == "rotate":
            heads, kv_heads, dim = rng.choice(LAYOUTS)
            c = dict(op=op, tokens=_log(rng, 1, 16384), heads=heads, kv_heads=kv_heads, dim=dim, rot=rng.choice((dim, dim, dim // 2, 16, 2 * rng.randint(1, dim // 2))),
                     interleaved=rng.random() < 0.5, norm=rng.random() < 0.75, far=_log(rng, 16, 1000000), dtype=rng.choice(("bf16", "fp16", "fp32")))
        elif op == "linear":
            q, p = rng.choice(LAYERS + ((_log(rng, 8, 16384), _log(rng, 8, 16384)), (8 * _log(rng, 8, 2048), 8 * _log(rng, 8, 2048))))
            group = rng.choice((0, 0, 64, 128, 256))
            c = dict(op=op, rows=rng.choice((_log(rng, 1, 64), _log(rng, 1, 4095))), q=q, p=p, bits=rng.choice((2, 3, 3, 4, 4, 4, 5, 6, 8)),
                     group=group, act=rng.choice(ACTS), bias=rng.random() < 0.5, residual=rng.random() < 0.5, dtype=dtype)
        else:
            heads, kv_heads, dim = rng.choice(LAYOUTS)
            seqs, q_hi = _log(rng, 1, 128), rng.choice((1, 1, 1, _log(rng, 2, 16), _log(rng, 16, 512)))
            own_hi = max(q_hi, _log(rng, 1, 4096))
            c = dict(op=op, seqs=seqs, idle=rng.choice((0, 0, rng.randint(0, seqs // 4))), q_lo=rng.randint(max(1, q_hi // 2), q_hi), q_hi=q_hi,
                     prefix=_log(rng, 1, 65536), own_lo=rng.randint(1, own_hi), own_hi=own_hi, heads=heads, kv_heads=kv_heads, dim=dim,
                     group=rng.choice([g for g in (32, 64, 128) if _padded(dim) % g == 0]), page=rng.choice((16, 32, 64, 128, 256)), dtype=dtype)
            if seqs * q_hi * heads * (c["prefix"] + own_hi) > 1 << 31 or seqs * own_hi * kv_heads * dim > 1 << 29:
                continue
        if _cost(c) <= most[op]:
            return c


def _cost(case):
    """Bytes or operations of the plain form, roughly: what a drawn case is held to."""
    w = work(case)
    if case["op"] == "grow":
        return case["seqs"] * (case["kv_hi"] + case["new_hi"])
    return w["bytes"] if case["op"] == "rotate" else w["flops"] + 200 * w["bytes"]


def _padded(dim):
    return 64 if dim <= 64 else 96 if dim <= 96 else 128


def _spread(n, lo, hi, off=0.0):
    """n whole numbers between lo and hi in a mixed order, from these alone; the last is hi."""
    v = [lo + int(round((((i + 1) * 0.6180339887 + off) % 1.0) * (hi - lo))) for i in range(n)]
    v[-1] = hi
    return v


# ---- grow ---------------------------------------------------------------------------------------------------------------

def _grow_lengths(case):
    new, kv = _spread(case["seqs"], case["new_lo"], case["new_hi"]), _spread(case["seqs"], case["kv_lo"], case["kv_hi"], 0.3)
    kv = [max(k, case["prefix"]) for k in kv]           # every sequence began behind the prefix
    ends = [0] * case["seqs"]
    for i in range(case["ends"]):                       # ended ones take no tokens in this step
        b = (7 + i * max(1, case["seqs"] // max(1, case["ends"]))) % case["seqs"]
        ends[b], new[b] = 1, 0
    return new, kv, ends


def _prepare_grow(case, seed, gen):
    dev, P, first = "cuda", case["page"], case["prefix"] // case["page"]
    new, kv, ends = _grow_lengths(case)
    held, grown = [-(-n // P) for n in kv], [-(-(n + m) // P) for n, m in zip(kv, new)]
    width, pages = max(1, max(grown)), sum(grown) + first + 7
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu()   # pages have been handed out in no order
    table = torch.full((len(kv), width), -1, dtype=torch.int32)
    table[:, :first] = order[:first]
    done = first
    for b, n in enumerate(held):
        table[b, first:n] = order[done:done + n - first]
        done += n - first
    at = int(torch.randint(pages, (1,), generator=gen, device=dev).item())          # where the ring's front has got to
    ring = torch.full((pages,), -1, dtype=torch.int32)
    ring[(at + torch.arange(pages - done)) % pages] = order[done:]
    as32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    most = sum(new) + 5                                 # the step's buffers hold a few tokens more than come
    st = dict(case=case, new=as32(new), kv_len=as32(kv), ends=torch.tensor(ends, dtype=torch.uint8, device=dev), table=table.to(dev),
              ring=ring.to(dev), state=as32([at, pages - done]), pages=pages, most=most)
    st.update(kv_out=torch.empty_like(st["kv_len"]), state_out=torch.empty_like(st["state"]))
    if own:
        from paper_2309_01885_gb300 import qe
        st["cache"] = qe.KVCache(pages, P, 1, 64, 64)
        st["pool"] = qe.PagePool(st["cache"], ring=st["ring"], state=st["state"])
        st["workspace"] = torch.empty(qe.qe_cache_grow_workspace(len(kv)), dtype=torch.uint8, device=dev)
        st["q_start"] = torch.empty(len(kv) + 1, dtype=torch.int32, device=dev)
        st["slots"] = torch.empty(most, dtype=torch.int64, device=dev)
        st["positions"] = torch.empty(most, dtype=torch.int32, device=dev)
    return st


def _grow(st):
    case, table, ring, pages = st["case"], st["table"], st["ring"], st["pages"]
    P, kept, dev = case["page"], case["prefix"] // case["page"], table.device
    n, length, ends = st["new"].long(), st["kv_len"].long(), st["ends"].bool()
    head, count = st["state"].long()
    start = torch.where(ends, case["prefix"], length)
    had, k0, k1 = (length + P - 1) // P, (start + P - 1) // P, (start + n + P - 1) // P
    need, back = k1 - k0, torch.where(ends, had - kept, 0)
    need_at, back_at = need.cumsum(0) - need, back.cumsum(0) - back
    q_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), n.cumsum(0)])
    k = torch.arange(table.shape[1], device=dev)
    # pages that come back go to the ring's end (a place behind the ring takes what is none of them)
    to = torch.where(ends[:, None] & (k >= kept) & (k < had[:, None]), (head + count + back_at[:, None] + k - kept) % pages, pages)
    bigger = torch.cat([ring, ring[:1]])
    bigger[to.flatten()] = table.flatten()
    taken = ring[(head + need_at[:, None] + k - k0[:, None]).remainder(pages)]
    table.copy_(torch.where((k >= k0[:, None]) & (k < k1[:, None]), taken, table))
    ring.copy_(bigger[:pages])
    i = torch.arange(st["most"], device=dev)
    b = torch.searchsorted(q_start[1:], i, right=True).clamp(max=len(n) - 1)
    live = i < q_start[-1]
    t = torch.where(live, start[b] + i - q_start[b], 0)
    slots = torch.where(live, table[b, t // P].long() * P + t % P, -1)
    st["kv_out"].copy_(start + n)
    st["state_out"].copy_(torch.stack([(head + need.sum()) % pages, count - need.sum() + back.sum()]))
    return q_start.to(torch.int32), slots, t.to(torch.int32), st["kv_out"], table, ring, st["state_out"]


def _exact_grow(case, seed):
    """One sequence and one token after the other."""
    st = prepare(case, seed)
    P, kept, pages = case["page"], case["prefix"] // case["page"], st["pages"]
    new, kv, ends = (st[k].cpu().tolist() for k in ("new", "kv_len", "ends"))
    table, ring, (head, count) = st["table"].cpu().numpy().copy(), st["ring"].cpu().numpy().copy(), st["state"].cpu().tolist()
    tail, q_start, slots, at = (head + count) % pages, [0], [], []
    for b, n in enumerate(new):
        if ends[b]:
            for k in range(kept, -(-kv[b] // P)):
                ring[tail] = table[b, k]
                tail, count = (tail + 1) % pages, count + 1
            kv[b] = case["prefix"]
        for _ in range(n):
            if kv[b] % P == 0:
                table[b, kv[b] // P] = ring[head]
                head, count = (head + 1) % pages, count - 1
            at.append(kv[b])
            slots.append(int(table[b, kv[b] // P]) * P + kv[b] % P)
            kv[b] += 1
        q_start.append(len(slots))
    rest = st["most"] - len(slots)
    give = lambda v, t: torch.as_tensor(np.asarray(v), device="cuda").to(t)
    return (give(q_start, torch.int32), give(slots + [-1] * rest, torch.int64), give(at + [0] * rest, torch.int32), give(kv, torch.int32),
            give(table, torch.int32), give(ring, torch.int32), give([head, count], torch.int32))


# ---- rotate -------------------------------------------------------------------------------------------------------------

THETA, EPS = 10000.0, 1e-5


def _prepare_rotate(case, seed, gen):
    dev, H, K, dim, n = "cuda", case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    dtype = DTYPES[case["dtype"]]
    # queries and keys lie inside the fused projection's output, as it leaves the product
    fused = torch.empty(n, H + 2 * K, dim, dtype=dtype, device=dev)
    loud = 1.0 + 3.0 * torch.rand(H + 2 * K, dim, generator=gen, device=dev)
    for a in range(0, n, 2048):
        fused[a:a + 2048] = torch.randn(min(2048, n - a), H + 2 * K, dim, generator=gen, device=dev) * loud
    st = dict(case=case, q=fused[:, :H], k=fused[:, H:H + K],
              positions=torch.randint(case["far"], (n,), generator=gen, device=dev, dtype=torch.int32), q_weight=None, k_weight=None)
    if case["norm"]:
        st["q_weight"], st["k_weight"] = ((1.0 + 0.3 * torch.randn(dim, generator=gen, device=dev)).to(dtype) for _ in range(2))
    if own:
        from paper_2309_01885_gb300 import qe
        st["rope"] = qe.Rope(case["rot"], theta=THETA, interleaved=case["interleaved"])
    return st


def _rotate(st):
    case, R = st["case"], st["case"]["rot"]
    i = torch.arange(R // 2, device=st["q"].device, dtype=torch.float64)
    angle = st["positions"].double()[:, None, None] * THETA ** (-2.0 * i / R)
    cos, sin = angle.cos().float(), angle.sin().float()
    found = []
    for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        a, b = (y[..., 0:R:2], y[..., 1:R:2]) if case["interleaved"] else (y[..., :R // 2], y[..., R // 2:R])
        turned = (a * cos - b * sin, b * cos + a * sin)
        turned = torch.stack(turned, -1).flatten(-2) if case["interleaved"] else torch.cat(turned, -1)
        found.append(torch.cat([turned, y[..., R:]], -1).to(x.dtype))
    return tuple(found)


def _exact_rotate(case, seed):
    st = prepare(case, seed)
    R, found = case["rot"], []
    place = np.arange(R // 2)
    first, second = (2 * place, 2 * place + 1) if case["interleaved"] else (place, place + R // 2)
    turn = torch.exp(torch.as_tensor(place, device="cuda").double() * (-2.0 * math.log(THETA) / R))
    for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for t in range(0, case["tokens"], 1024):
            y = x[t:t + 1024].double()
            if w is not None:
                y = y / (y.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * w.double()
            z = torch.complex(y[..., first], y[..., second])
            z = z * torch.polar(torch.ones_like(turn), st["positions"][t:t + 1024, None].double() * turn)[:, None]
            y[..., first], y[..., second] = z.real, z.imag
            out[t:t + 1024] = y
        found.append(out)
    return tuple(found)


# ---- linear -------------------------------------------------------------------------------------------------------------

def _prepare_linear(case, seed, gen):
    dev, q, p, n, dtype = "cuda", case["q"], case["p"], case["rows"], DTYPES[case["dtype"]]
    groups, top = (-(-p // case["group"]) if case["group"] else 1), 2 ** case["bits"] - 1
    # trained weights fill the middle of their grid: codes about its centre, as the quantizer leaves them
    codes = torch.empty(q, p, dtype=torch.uint8, device=dev)
    for a in range(0, q, 2048):
        codes[a:a + 2048] = (torch.randn(min(2048, q - a), p, generator=gen, device=dev) * (top / 6.0) + top / 2.0).round_().clamp_(0, top).to(torch.uint8)
    scales = (0.5 + torch.rand(q, groups, generator=gen, device=dev)) * (6.0 / (top * math.sqrt(p)))
    zeros = (torch.randn(q, groups, generator=gen, device=dev) * (top / 16.0) + top / 2.0).round_().clamp_(0, top)
    # a few input channels are loud, as they are in trained models
    x = torch.randn(n, p, generator=gen, device=dev)
    x *= 1.0 + 19.0 * (torch.rand(p, generator=gen, device=dev) < 0.005)
    st = dict(case=case, codes=codes, scales=scales, zeros=zeros, x=x.to(dtype), bias=None, residual=None)
    if case["bias"]:
        st["bias"] = (0.5 * torch.randn(q, generator=gen, device=dev)).to(dtype)
    if case["residual"]:
        st["residual"] = torch.randn(n, q, generator=gen, device=dev).to(dtype)
    if own:  # the weights as a program holds them, and its workspace
        from paper_2309_01885_gb300 import qe
        st["weights"] = qe.QuantizedWeights(codes, scales if case["group"] else scales[:, 0].contiguous(),
                                            zeros if case["group"] else zeros[:, 0].contiguous(), case["bits"], group_size=case["group"])
        st["workspace"] = torch.empty(qe.qe_linear_workspace(st["weights"], n), dtype=torch.uint8, device=dev)
    return st


def _act(y, name):
    if name == "relu":
        return y.clamp(min=0.0)
    if name == "silu":
        return y / (1.0 + (-y).exp())
    if name == "gelu":
        return y * 0.5 * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return y * 0.5 * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    return y


def _linear(st):
    case, p = st["case"], st["case"]["p"]
    G = case["group"] or p
    grid = lambda v: v if v.shape[1] == 1 else v.repeat_interleave(G, 1)[:, :p]
    w = st["codes"].float().sub_(grid(st["zeros"])).mul_(grid(st["scales"]))
    y = st["x"].float() @ w.T
    if st["bias"] is not None:
        y = y + st["bias"].float()
    y = _act(y, case["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(st["x"].dtype)


def _exact_linear(case, seed):
    if work(case)["flops"] > 1.5e12:
        return None
    st = prepare(case, seed)
    x, G = st["x"].double(), case["group"] or case["p"]
    y = torch.zeros(case["rows"], case["q"], dtype=torch.float64, device="cuda")
    for a in range(0, case["q"], 2048):
        part = slice(a, a + 2048)
        for g in range(st["scales"].shape[1]):
            cols = slice(g * G, min((g + 1) * G, case["p"]))
            step = st["codes"][part, cols].double() - st["zeros"][part, g, None].double()
            y[:, part] += (x[:, cols] @ step.T) * st["scales"][part, g].double()
    if case["bias"]:
        y += st["bias"].double()
    if case["act"] == "relu":
        y = torch.maximum(y, torch.zeros_like(y))
    elif case["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif case["act"] == "gelu":
        y = 0.5 * y * torch.erfc(-y / math.sqrt(2.0))
    elif case["act"] == "gelu_tanh":
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    return y + st["residual"].double() if case["residual"] else y


# ---- shared -------------------------------------------------------------------------------------------------------------

def _shared_lengths(case):
    """(query rows, own tokens) of each sequence; idle places have a row and hold nothing, not even the prefix."""
    q = _spread(case["seqs"], case["q_lo"], case["q_hi"], 0.7)
    mine = [max(n, m) for n, m in zip(q, _spread(case["seqs"], case["own_lo"], case["own_hi"]))]
    for b in range(case["idle"]):
        q[3 * b % case["seqs"]], mine[3 * b % case["seqs"]] = 1, -1
    return q, mine


def _views(st):
    """The cache's parts: key words, value halfwords, key grids, value grids."""
    c, D = st["case"], _padded(st["case"]["dim"])
    P, H, G, C = c["page"], c["kv_heads"], _padded(c["dim"]) // c["group"], _padded(c["dim"]) // 32
    codes, grids = P * D // 2, P * G * 4
    b = st["data"].view(-1, H, 2 * codes + 2 * grids)
    k = b[..., :codes].view(torch.int32).unflatten(-1, (P // 8, 8, 4, C))
    v = b[..., codes:2 * codes].view(torch.int16).unflatten(-1, (P // 8, 8, 4, C, 2))
    kg = b[..., 2 * codes:2 * codes + grids].view(torch.int32).unflatten(-1, (P, G))
    vg = b[..., 2 * codes + grids:].view(torch.int32).unflatten(-1, (P, G))
    return k, v, kg, vg


def _quantize(x, case):
    """Codes [tokens, heads, D] and grid words [tokens, heads, groups] of x [tokens, heads, dim]."""
    x = torch.nn.functional.pad(x.float(), (0, _padded(case["dim"]) - case["dim"])).unflatten(-1, (-1, case["group"]))
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    s = ((hi - lo) / torch.full_like(hi, 15.0)).to(torch.bfloat16).float().clamp(min=2.0 ** -126)
    z = torch.round(lo.abs() / s)
    code = (torch.round(x / s[..., None]) + z[..., None]).clamp(0.0, 15.0).to(torch.int32).flatten(-2)
    return code, s.view(torch.int32) | (z.view(torch.int32) >> 16)


def _write(st, k, v, slots):
    case = st["case"]
    kw, vh, kg, vg = _views(st)
    page, tok = slots // case["page"], slots % case["page"]
    kc, kgrid = _quantize(k, case)
    vc, vgrid = _quantize(v, case)
    bit = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device=kc.device, dtype=torch.int32)
    kword = (kc.unflatten(-1, (-1, 4, 4, 2)) << bit).sum((-2, -1)).to(torch.int32)              # [n, H, w, t]
    vhalf = (vc.unflatten(-1, (-1, 8, 4)) << bit[:, 0]).sum(-1).to(torch.int16)                 # [n, H, w, r]
    kw[page, :, tok // 8, tok % 8] = kword.transpose(-1, -2)
    t, h = tok % 8 // 2, tok % 2
    vh.permute(0, 2, 4, 6, 1, 3, 5)[page, tok // 8, t, h] = vhalf.transpose(-1, -2)
    kg[page, :, tok], vg[page, :, tok] = kgrid, vgrid


def _values(code, word, case):
    """s (c - z) in binary32, [..., dim], from codes [..., D] and grid words [..., groups]."""
    s, z = (word & -65536).view(torch.float32), (word << 16).view(torch.float32)
    x = s[..., None] * (code.unflatten(-1, (-1, case["group"])).float() - z[..., None])
    return x.flatten(-2)[..., :case["dim"]]


def _read(st, slots):
    """Keys and values [..., heads, dim] of the slots, in binary32."""
    case = st["case"]
    kw, vh, kg, vg = _views(st)
    page, tok = slots // case["page"], slots % case["page"]
    bit = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=slots.device, dtype=torch.int32)
    kc = (kw.permute(0, 2, 3, 1, 5, 4)[page, tok // 8, tok % 8][..., None] >> bit) & 15         # [.., H, w, t, 8]
    vq = vh.permute(0, 2, 4, 6, 1, 5, 3)[page, tok // 8, tok % 8 // 2, tok % 2].to(torch.int32)  # [.., H, w, r]
    vc = (vq[..., None] >> bit[:8:2]) & 15
    kg, vg = kg.transpose(1, 2)[page, tok], vg.transpose(1, 2)[page, tok]
    return _values(kc.flatten(-3), kg, case), _values(vc.flatten(-3), vg, case)


def _prepare_shared(case, seed, gen):
    dev = "cuda"

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32)

    H, dim, P, D, first = case["kv_heads"], case["dim"], case["page"], _padded(case["dim"]), case["prefix"]
    q_len, mine = _shared_lengths(case)
    kv_len = [first + m if m >= 0 else 0 for m in mine]
    full = -(-first // P)
    # own tokens begin inside the prefix's last page where that is not full: each sequence has a page of its own there
    need = [max(0, -(-n // P) - first // P) for n in kv_len]
    width, pages = max(1, max([full] + [-(-n // P) for n in kv_len])), full + sum(need) + 2
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu()
    table, done = torch.zeros(len(kv_len), width, dtype=torch.int32), full
    for b, n in enumerate(need):
        if kv_len[b]:
            table[b, :first // P] = order[:first // P]
            table[b, first // P:first // P + n] = order[done:done + n]
        done += n
    block = P * D + 2 * P * (D // case["group"]) * 4
    st = dict(case=case, data=torch.zeros(pages * H * block, dtype=torch.uint8, device=dev))
    far = normal(H, dim) * (torch.rand(H, dim, generator=gen, device=dev) < 0.04) * 4.0
    st.update(prefix_pages=order[:full].to(dev), page_table=table.to(dev))
    for b in range(-1, len(kv_len)):                   # the cache as earlier steps have left it: the prefix, then what follows
        row = st["prefix_pages"] if b < 0 else st["page_table"][b]
        begin, end = (0, first) if b < 0 else (first, kv_len[b])
        for a in range(begin, end, 16384):
            j = torch.arange(a, min(end, a + 16384), device=dev)
            _write(st, normal(len(j), H, dim) + far, 0.5 * normal(len(j), H, dim), row[j // P].long() * P + j % P)
    st.update(q=(1.2 * normal(sum(q_len), case["heads"], dim)).to(DTYPES[case["dtype"]]),
              q_start=torch.tensor([0] + q_len, device=dev).cumsum(0).to(torch.int32),
              kv_len=torch.tensor(kv_len, dtype=torch.int32, device=dev), max_q=max(q_len), max_kv=max(1, max(kv_len)))
    if own:
        from paper_2309_01885_gb300 import qe
        st["cache"] = qe.KVCache(pages, P, H, dim, case["group"], data=st["data"])
        n = qe.qe_cache_attention_shared_workspace(st["cache"], len(q_len), case["heads"], sum(q_len), st["max_q"], st["max_kv"], first)
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device=dev)
    return st


def _shared(st):
    """Scores over the prefix, computed for all sequences at once, and over each one's own tokens, padded to the longest."""
    case, q, start, kv = st["case"], st["q"], st["q_start"].long(), st["kv_len"].long()
    H, g, n, first, P = case["kv_heads"], case["heads"] // case["kv_heads"], st["max_q"], case["prefix"], case["page"]
    dev, m = q.device, max(1, st["max_kv"] - case["prefix"])
    row, tok, j0 = torch.arange(n, device=dev), torch.arange(m, device=dev) + first, torch.arange(first, device=dev)
    rows = start[1:] - start[:-1]
    live = row < rows[:, None]
    x = q[(start[:-1, None] + row).clamp(max=q.shape[0] - 1)].float()                            # [B, n, heads, dim]
    x = x.unflatten(2, (H, g)).permute(0, 2, 1, 3, 4).flatten(2, 3) * (1.0 / math.sqrt(case["dim"]))   # [B, H, n g, dim]
    page = st["page_table"][:, (tok // P).clamp(max=st["page_table"].shape[1] - 1)].long()
    k0, v0 = _read(st, st["prefix_pages"][j0 // P].long() * P + j0 % P)                          # [prefix, H, dim]
    k1, v1 = _read(st, page * P + tok % P)                                                       # [B, m, H, dim]
    at = ((kv - rows)[:, None] + row).repeat_interleave(g, 1)[:, None, :, None]                  # [B, 1, n g, 1]
    s0 = (x @ k0.permute(1, 2, 0)).masked_fill_(j0 > at, -math.inf)
    s1 = (x @ k1.permute(0, 2, 3, 1)).masked_fill_((tok > at) | (tok >= kv[:, None, None, None]), -math.inf)
    top = torch.maximum(s0.amax(-1, keepdim=True), s1.amax(-1, keepdim=True))
    top = torch.where(top > -math.inf, top, 0.0)
    s0, s1 = s0.sub_(top).exp_(), s1.sub_(top).exp_()
    total = s0.sum(-1, keepdim=True) + s1.sum(-1, keepdim=True)
    v1 = torch.where((tok < kv[:, None])[..., None, None], v1, 0.0)
    out = (s0 @ v0.permute(1, 0, 2) + s1 @ v1.permute(0, 2, 1, 3)) / torch.where(total > 0.0, total, 1.0)
    return out.unflatten(2, (n, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)[live].to(q.dtype)


def _exact_cell(st, slot):
    """Keys and values [n, heads, dim] in binary64 that the cache's bytes stand for at the slots, channel by channel."""
    c, dev = st["case"], slot.device
    D, P, H, g = _padded(c["dim"]), c["page"], c["kv_heads"], c["group"]
    word = st["data"].view(torch.int32).long() & 0xFFFFFFFF
    size = (P * D + 8 * P * (D // g)) // 4                                # words of a page's head
    head, ch = torch.arange(H, device=dev)[:, None], torch.arange(c["dim"], device=dev)
    base = ((slot // P)[:, None, None] * H + head) * size
    j = (slot % P)[:, None, None]
    chunk, inner = ch // 32, ch % 32
    at_k = base + (j // 8) * D + (4 * (j % 8) + inner // 8) * (D // 32) + chunk
    bit_k = 4 * (inner % 8 // 2) + 16 * (inner % 2)
    at_v = base + P * D // 8 + (j // 8) * D + (4 * (inner // 4) + j % 8 // 2) * (D // 32) + chunk
    bit_v = 4 * (inner % 4) + 16 * (j % 2)
    at_g = base + P * D // 4 + j * (D // g) + ch // g
    found = []
    for at, bit, grid in ((at_k, bit_k, at_g), (at_v, bit_v, at_g + P * (D // g))):
        code, w = ((word[at] >> bit) & 15).double(), word[grid]
        scale = (w & 0xFFFF0000).to(torch.int32).view(torch.float32).double()
        zero = ((w & 0xFFFF) << 16).to(torch.int32).view(torch.float32).double()
        found.append(scale * (code - zero))
    return found


def _exact_shared(case, seed):
    if work(case)["flops"] > 1.5e12:
        return None
    st = prepare(case, seed)
    (q_len, mine), P, first = _shared_lengths(case), case["page"], case["prefix"]
    g, out, at = case["heads"] // case["kv_heads"], torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"), 0

    def cells(row, begin, end):
        j = torch.arange(begin, end, device="cuda")
        slots = row[j // P].long() * P + j % P
        return [torch.cat(x) for x in zip(*(_exact_cell(st, s) for s in slots.split(4096)))]

    k0, v0 = cells(st["prefix_pages"], 0, first)
    for b, (n, m) in enumerate(zip(q_len, mine)):
        if m >= 0:
            k1, v1 = cells(st["page_table"][b], first, first + m)
            hidden = torch.arange(m, device="cuda") > torch.arange(m - n, m, device="cuda")[:, None]
            for h in range(case["heads"]):
                x = st["q"][at:at + n, h].double() / math.sqrt(case["dim"])
                s = torch.cat([x @ k0[:, h // g].T, (x @ k1[:, h // g].T).masked_fill(hidden, -math.inf)], 1)
                p = torch.softmax(s, -1)
                out[at:at + n, h] = p[:, :first] @ v0[:, h // g] + p[:, first:] @ v1[:, h // g]
        at += n
    return out


# ---- all of them --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    return dict(grow=_prepare_grow, rotate=_prepare_rotate, linear=_prepare_linear, shared=_prepare_shared)[case["op"]](case, seed, gen)


def run(st):
    case = st["case"]
    if not own:
        return dict(grow=_grow, rotate=_rotate, linear=_linear, shared=_shared)[case["op"]](st)
    from paper_2309_01885_gb300 import qe
    if case["op"] == "grow":
        qe.qe_cache_grow(st["cache"], st["pool"], st["kv_len"], st["new"], st["table"], st["most"], ends=st["ends"], prefix=case["prefix"],
                         kv_len_out=st["kv_out"], state_out=st["state_out"], q_start=st["q_start"], slots=st["slots"],
                         positions=st["positions"], workspace=st["workspace"])
        return st["q_start"], st["slots"], st["positions"], st["kv_out"], st["table"], st["ring"], st["state_out"]
    if case["op"] == "rotate":
        return qe.qe_norm_rotate(st["q"], st["k"], st["positions"], st["rope"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS)
    if case["op"] == "linear":
        return qe.qe_linear(st["weights"], st["x"], bias=st["bias"], activation=case["act"], residual=st["residual"], workspace=st["workspace"])
    return qe.qe_cache_attention_shared(st["cache"], st["q"], st["q_start"], st["kv_len"], st["page_table"], st["max_q"], st["max_kv"],
                                        st["prefix_pages"], case["prefix"], workspace=st["workspace"])


def work(case):
    if case["op"] == "grow":
        new, kv, ends = _grow_lengths(case)
        P = case["page"]
        moved = sum(-(-(k + n) // P) + -(-k // P) * e - -(-k // P) for n, k, e in zip(new, kv, ends))
        return dict(bytes=case["seqs"] * (4 + 4 + 1 + 4 + 4) + 12 * sum(new) + 8 * max(0, moved), flops=case["seqs"] * 8 + 6 * sum(new))
    size = SIZE[case["dtype"]]
    if case["op"] == "rotate":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return dict(bytes=2 * n * size + 4 * case["tokens"], flops=7 * n)
    if case["op"] == "linear":
        q, p, n = case["q"], case["p"], case["rows"]
        groups = -(-p // case["group"]) if case["group"] else 1
        return dict(bytes=-(-q * p * case["bits"] // 8) + q * groups * 5 + n * (p + q * (2 if case["residual"] else 1)) * size,
                    flops=2 * n * q * p)
    D = _padded(case["dim"])
    token = case["kv_heads"] * (D + 8 * (D // case["group"]))             # bytes of a cached token, keys and values
    q_len, mine = _shared_lengths(case)
    pairs = sum(n * (case["prefix"] + m) - n * (n - 1) // 2 for n, m in zip(q_len, mine) if m >= 0)
    seen = case["prefix"] + sum(m for m in mine if m > 0)
    return dict(bytes=seen * token + 2 * sum(q_len) * case["heads"] * case["dim"] * size, flops=4 * case["dim"] * case["heads"] * pairs)


def exact(case, seed):
    return dict(grow=_exact_grow, rotate=_exact_rotate, linear=_exact_linear, shared=_exact_shared)[case["op"]](case, seed)
