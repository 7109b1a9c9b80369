"""The serving step's C ABI without a GPU: sizes, refusals, and the ctypes mirrors of its structs."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2309_01885_gb300 import build, qe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("name,mirror", [("qe_growth", qe.QEGrowth), ("qe_rope", qe.QERope), ("qe_heads", qe.QEHeads),
                                         ("qe_layer", qe.QELayer), ("qe_product", qe.QEProduct)])
def test_structs_match_header(tmp_path, name, mirror):
    fields = [f[0] for f in mirror._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include "qe.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) {\n'
                   f'    printf("%zu\\n", sizeof({name}));\n'
                   + "".join(f'    printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "    return 0;\n}\n")
    exe = tmp_path / "s"
    subprocess.check_call(["gcc", "-std=c11", f"-I{os.path.join(ROOT, 'include')}", "-o", str(exe), str(src)])
    out = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    assert out == [ctypes.sizeof(mirror)] + [getattr(mirror, f).offset for f in fields]


@pytest.mark.parametrize("packed,mirror", [(qe._GROWTH, qe.QEGrowth), (qe._HEADS, qe.QEHeads), (qe._PRODUCT, qe.QEProduct)])
def test_packed_structs_match_their_mirrors(packed, mirror):
    """Field by field: a number in one of them comes out of the mirror under its name, and nowhere else."""
    assert packed.size <= ctypes.sizeof(mirror) <= packed.size + 4
    for i, (name, kind) in enumerate(mirror._fields_):
        values = [0.0 if k is ctypes.c_float else 0 for _, k in mirror._fields_]
        values[i] = 2.0 if kind is ctypes.c_float else 77
        got = mirror.from_buffer_copy(packed.pack(*values) + b"\0" * 8)
        assert {n: getattr(got, n) or 0 for n, _ in mirror._fields_} == {n: v for (n, _), v in zip(mirror._fields_, values)}


def filled(struct, values):
    s = struct()
    for k, v in values.items():
        setattr(s, k, v)
    return s


CACHE = qe.QECache(0x100000, 1 << 40, 4, 64, 2, 128, 32)


# ---- grow ----

GROWTH = dict(seqs=3, max_tokens=10, prefix=64, table_ld=4, new_tokens=0x1000, ends=None, kv_len=0x2000, kv_len_out=0x2000, page_table=0x3000,
              ring=0x4000, state=0x5000, state_out=0x5000, q_start=0x6000, slots=0x7000, positions=None)


def test_grow_refuses(lib):
    def call(ws=0x100000, ws_bytes=1 << 20, **kw):
        gr = filled(qe.QEGrowth, {**GROWTH, **kw})
        return lib.qe_cache_grow(ctypes.addressof(CACHE), ctypes.addressof(gr), ws, ws_bytes, None)

    for bad in (dict(seqs=0), dict(seqs=65536), dict(max_tokens=-1), dict(max_tokens=(1 << 30) + 1), dict(prefix=-64), dict(prefix=63),
                dict(prefix=5 * 64), dict(prefix=1 << 31), dict(table_ld=0), dict(table_ld=1 << 30), dict(new_tokens=None), dict(kv_len=None),
                dict(kv_len_out=None), dict(page_table=None), dict(ring=None), dict(state=None), dict(state_out=None), dict(q_start=None),
                dict(slots=None), dict(new_tokens=0x1002), dict(slots=0x7004), dict(positions=0x7001), dict(ws=0x100010)):
        assert call(**bad) == qe.QE_ERR_INVALID_ARG, bad
    assert call(ws_bytes=100) == qe.QE_ERR_OOM
    gr = filled(qe.QEGrowth, GROWTH)
    assert lib.qe_cache_grow(None, ctypes.addressof(gr), None, 0, None) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_cache_grow(ctypes.addressof(CACHE), None, None, 0, None) == qe.QE_ERR_INVALID_ARG
    odd = qe.QECache(0x100000, 1 << 40, 4, 48, 2, 128, 32)
    assert lib.qe_cache_grow(ctypes.addressof(odd), ctypes.addressof(gr), None, 0, None) == qe.QE_ERR_UNSUPPORTED


def test_grow_workspace():
    assert qe.qe_cache_grow_workspace(1) <= qe.qe_cache_grow_workspace(1000) <= qe.qe_cache_grow_workspace(65535)
    for bad in (0, -1, 65536):
        with pytest.raises(qe.QEError):
            qe.qe_cache_grow_workspace(bad)


# ---- rotation ----

def test_rope_holds_turns():
    freq = [1.0, 0.25, 2.0 * math.pi * 0.75, -2.0 * math.pi * 0.25, 0.0, 7.0]
    r = qe.Rope(12, inv_freq=freq, interleaved=True)
    assert r._c.pairs == 6 and r._c.interleaved == 1
    for f, t in zip(freq, r._c.turns):
        want = f / (2.0 * math.pi) % 1.0
        off = abs(t / 2.0 ** 64 - want)
        assert min(off, 1.0 - off) <= 2.0 ** -52
    assert list(r._c.turns)[6:] == [0] * 122
    d = qe.Rope(128)
    assert abs(d._c.turns[63] / 2.0 ** 64 - 10000.0 ** (-126 / 128) / (2 * math.pi)) < 2.0 ** -55


def test_rope_refuses(lib):
    for bad in (dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=8, theta=0.0), dict(rotary_dim=8, inv_freq=[1.0])):
        with pytest.raises(ValueError):
            qe.Rope(**bad)
    for bad in (dict(rotary_dim=258), dict(rotary_dim=4, inv_freq=[1.0, math.inf]), dict(rotary_dim=4, inv_freq=[math.nan, 1.0])):
        with pytest.raises(qe.QEError):
            qe.Rope(**bad)
    assert lib.qe_rope_init(None, 4, 0, ctypes.addressof(qe.QERope())) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_rope_init((ctypes.c_double * 1)(1.0), 1, 0, None) == qe.QE_ERR_INVALID_ARG


def test_norm_rotate_refuses(lib):
    rope = qe.Rope(64)
    ok = dict(tokens=5, q_heads=4, k_heads=2, head_dim=64, dtype=qe.QE_BF16, weight_dtype=qe.QE_F32, Q=0x1000, K=0x2000, q_token=256, q_head=64,
              k_token=128, k_head=64, q_out=0x3000, k_out=0x4000, qo_token=256, qo_head=64, ko_token=128, ko_head=64, q_weight=0x5000,
              k_weight=0x6000, eps=1e-6, positions=0x7000, rope=rope._ref)

    def call(**kw):
        h = filled(qe.QEHeads, {**ok, **kw})
        return lib.qe_norm_rotate(ctypes.addressof(h), None)

    wide = qe.Rope(66)
    for bad in (dict(tokens=-1), dict(tokens=1 << 31), dict(q_heads=-1), dict(k_heads=65536), dict(head_dim=0), dict(dtype=3), dict(dtype=-1),
                dict(weight_dtype=9), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(rope=wide._ref), dict(Q=None), dict(k_out=None),
                dict(Q=0x1001), dict(dtype=qe.QE_F32, K=0x2002), dict(q_weight=0x5002), dict(positions=None), dict(positions=0x7002)):
        assert call(**bad) == qe.QE_ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=12), dict(head_dim=264)):
        assert call(**bad) == qe.QE_ERR_UNSUPPORTED, bad
    assert lib.qe_norm_rotate(None, None) == qe.QE_ERR_INVALID_ARG
    assert call(tokens=0, Q=None) == qe.QE_OK and call(q_heads=0, k_heads=0, Q=None) == qe.QE_OK


def test_norm_rotate_python_refuses(monkeypatch):
    x = torch.zeros(3, 4, 64)
    with pytest.raises(ValueError):                      # not on a device
        qe.qe_norm_rotate(x, x)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(qe, "_current_device", lambda: 0)
    x, pos, rope = torch.zeros(3, 4, 64), torch.zeros(3, dtype=torch.int32), qe.Rope(64)
    for bad in (dict(q=None, k=None), dict(q=x[0], k=None), dict(q=x, k=torch.zeros(2, 4, 64)), dict(q=x, k=x.half()),
                dict(q=x, k=x.transpose(1, 2).contiguous().transpose(1, 2)), dict(q=x, k=None, positions=None),
                dict(q=x, k=None, positions=pos.long()), dict(q=x, k=None, positions=pos[:2]), dict(q=x, k=None, k_weight=torch.ones(64)),
                dict(q=x, k=None, q_weight=torch.ones(63)), dict(q=x, k=x, q_weight=torch.ones(64), k_weight=torch.ones(64).half()),
                dict(q=x, k=None, q_out=x[:, :2])):
        with pytest.raises(ValueError):
            qe.qe_norm_rotate(**{**dict(positions=pos, rope=rope), **bad})


# ---- products ----

@pytest.mark.parametrize("bits,stored", [(2, 2), (3, 3), (4, 4), (5, 8), (6, 8), (7, 8), (8, 8)])
def test_linear_size(bits, stored):
    up = lambda n: -(-n // 256) * 256
    for q, p, group in ((1, 1, 0), (16, 64, 0), (17, 65, 64), (4096, 4096, 128), (14848, 59392, 0), (768, 768, 768)):
        tiles, units = -(-q // 16), -(-p // 64)
        groups = -(-p // group) if 0 < group < p else 1
        grids = tiles * groups * 16
        assert qe.qe_linear_size(q, p, bits, group) == up(tiles * units * 128 * stored) + up(4 * grids) + up(-(-tiles // 2) * 2 * groups * 16)


def test_linear_size_refuses(lib):
    for bad in (dict(q=0), dict(p=0), dict(q=(1 << 24) + 1), dict(p=(1 << 24) + 1), dict(bits=1), dict(bits=9), dict(group_size=-64)):
        with pytest.raises(qe.QEError) as e:
            qe.qe_linear_size(**{**dict(q=64, p=256, bits=4, group_size=64), **bad})
        assert e.value.status == qe.QE_ERR_INVALID_ARG, bad
    for group in (32, 100):
        with pytest.raises(qe.QEError) as e:
            qe.qe_linear_size(64, 256, 4, group)
        assert e.value.status == qe.QE_ERR_UNSUPPORTED
    assert lib.qe_linear_size(4, 4, 4, 0, None) == qe.QE_ERR_INVALID_ARG


def test_linear_refuses(lib):
    need = qe.qe_linear_size(100, 200, 4, 64)
    shape = dict(data=0x100000, bytes=need, q=100, p=200, bits=4, group_size=64)
    ok = dict(rows=5, dtype=qe.QE_BF16, bias_dtype=qe.QE_F32, X=0x1000, ldx=200, bias=0x2000, act=0, residual=0x3000, ldr=100, Y=0x4000, ldy=100)

    def call(layer=None, ws=0x100000, ws_bytes=1 << 20, **kw):
        a, b = filled(qe.QELayer, {**shape, **(layer or {})}), filled(qe.QEProduct, {**ok, **kw})
        return lib.qe_linear(ctypes.addressof(a), ctypes.addressof(b), ws, ws_bytes, None)

    def pack(layer=None, codes=0x1000, ldc=200, scales=0x2000, zeros=0x3000):
        a = filled(qe.QELayer, {**shape, **(layer or {})})
        return lib.qe_linear_pack(ctypes.addressof(a), codes, ldc, scales, zeros, None)

    for bad in (dict(data=None), dict(data=0x100080), dict(bytes=need - 1), dict(q=0), dict(bits=1), dict(group_size=-1)):
        assert call(layer=bad) == qe.QE_ERR_INVALID_ARG and pack(layer=bad) == qe.QE_ERR_INVALID_ARG, bad
    assert call(layer=dict(group_size=32)) == qe.QE_ERR_UNSUPPORTED
    for bad in (dict(codes=None), dict(scales=None), dict(zeros=None), dict(ldc=199), dict(scales=0x2002)):
        assert pack(**bad) == qe.QE_ERR_INVALID_ARG, bad
    for bad in (dict(rows=-1), dict(rows=1 << 31), dict(dtype=5), dict(act=-1), dict(act=5), dict(bias_dtype=7), dict(X=None), dict(Y=None),
                dict(ldx=199), dict(ldy=99), dict(ldr=99), dict(X=0x1001), dict(Y=0x4001), dict(residual=0x3001), dict(bias=0x2002), dict(ws=0x100010)):
        assert call(**bad) == qe.QE_ERR_INVALID_ARG, bad
    assert call(dtype=qe.QE_F32) == qe.QE_ERR_UNSUPPORTED
    assert call(rows=0, X=None, Y=None) == qe.QE_OK
    a, n = filled(qe.QELayer, shape), ctypes.c_size_t(0)
    assert lib.qe_linear(ctypes.addressof(a), None, None, 0, None) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_linear_workspace(None, 5, ctypes.byref(n)) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_linear_workspace(ctypes.addressof(a), -1, ctypes.byref(n)) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_linear_workspace(ctypes.addressof(a), 5, None) == qe.QE_ERR_INVALID_ARG


# ---- attention behind a shared prefix ----

AT = dict(seqs=3, rows=3, q_heads=8, causal=1, window=0, scale=0.0, max_q=1, max_kv=100, q_start=0x1000, kv_len=0x2000, page_table=0x3000, table_ld=2)


def test_shared_refuses(lib):
    def call(pages=0x8000, prefix=70, Q=0x4000, ws=0x100000, ws_bytes=1 << 30, **kw):
        at = filled(qe.QEAttention, {**AT, **kw})
        return lib.qe_cache_attention_shared(ctypes.addressof(CACHE), ctypes.addressof(at), pages, prefix, Q, 1024, 128, 0x5000, 1024, 128,
                                             qe.QE_BF16, None, ws, ws_bytes, None)

    for bad in (dict(pages=None), dict(pages=0x8002), dict(prefix=-1), dict(prefix=(1 << 30) + 1), dict(seqs=0), dict(q_heads=7), dict(Q=None),
                dict(kv_len=None), dict(max_q=4), dict(ws=0x100010)):
        assert call(**bad) == qe.QE_ERR_INVALID_ARG, bad
    assert call(window=5) == qe.QE_ERR_UNSUPPORTED
    assert call(rows=0, max_q=0) == qe.QE_OK
    assert lib.qe_cache_attention_shared(ctypes.addressof(CACHE), None, 0x8000, 70, 0x4000, 1024, 128, 0x5000, 1024, 128, qe.QE_BF16, None, None,
                                         0, None) == qe.QE_ERR_INVALID_ARG
    at, n = filled(qe.QEAttention, AT), ctypes.c_size_t(0)
    assert lib.qe_cache_attention_shared_workspace(ctypes.addressof(CACHE), ctypes.addressof(at), 70, None) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_cache_attention_shared_workspace(ctypes.addressof(CACHE), ctypes.addressof(at), -1, ctypes.byref(n)) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_cache_attention_shared_workspace(ctypes.addressof(CACHE), ctypes.addressof(at), 70, ctypes.byref(n)) == qe.QE_OK
    assert n.value >= 3 * 8 * (128 + 2) * 4
