"""The key/value cache's C ABI without a GPU: sizes, refusals, and the ctypes mirrors of its structs."""
import ctypes
import os
import subprocess

import pytest

from paper_2309_01885_gb300 import build, qe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_lib()
    return qe.load()


def _fake(n=1):
    return 0x1000 * n            # never dereferenced: rejected before any launch


@pytest.mark.parametrize("name,mirror", [("qe_cache", qe.QECache), ("qe_attention", qe.QEAttention)])
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


@pytest.mark.parametrize("dim,group,token", [(128, 32, 160), (128, 64, 144), (128, 128, 136), (64, 32, 80), (64, 64, 72),
                                             (96, 32, 120), (80, 32, 120), (72, 32, 120), (8, 64, 72), (120, 128, 136)])
def test_size(dim, group, token):
    """Keys and values: half a byte a channel and a word a group, each."""
    for pages, page, heads in ((1, 16, 1), (7, 64, 8), (1 << 20, 256, 32)):
        assert qe.qe_cache_size(pages, page, heads, dim, group) == pages * page * heads * token


def test_size_refuses():
    ok = dict(pages=4, page_size=64, kv_heads=8, head_dim=128, group_size=32)
    for bad in (dict(pages=0), dict(pages=-1), dict(pages=1 << 31), dict(page_size=0), dict(kv_heads=0), dict(kv_heads=65536),
                dict(head_dim=0), dict(group_size=0)):
        with pytest.raises(qe.QEError) as e:
            qe.qe_cache_size(**{**ok, **bad})
        assert e.value.status == qe.QE_ERR_INVALID_ARG, bad
    for bad in (dict(page_size=8), dict(page_size=48), dict(page_size=1 << 17), dict(head_dim=4), dict(head_dim=100),
                dict(head_dim=136), dict(group_size=16), dict(group_size=48), dict(head_dim=96, group_size=64),
                dict(head_dim=64, group_size=128)):
        with pytest.raises(qe.QEError) as e:
            qe.qe_cache_size(**{**ok, **bad})
        assert e.value.status == qe.QE_ERR_UNSUPPORTED, bad


def _cache(**kw):
    f = dict(data=0x100000, bytes=1 << 40, pages=4, page_size=64, kv_heads=2, head_dim=128, group_size=32)
    f.update(kw)
    return qe.QECache(*[f[n] for n, _ in qe.QECache._fields_])


BAD_CACHES = [dict(data=None), dict(data=0x100010), dict(bytes=4 * 64 * 2 * 160 - 1), dict(pages=0)]


def test_append_and_read_refuse(lib):
    ok = dict(K=_fake(), V=_fake(2), slots=_fake(3), n=5, dtype=qe.QE_BF16)

    def append(c, **kw):
        a = {**ok, **kw}
        return lib.qe_cache_append(c and ctypes.addressof(c), a["K"], 256, 128, a["V"], 256, 128, a["dtype"], a["slots"], a["n"], None)

    def read(c, **kw):
        a = {**ok, **kw}
        return lib.qe_cache_read(c and ctypes.addressof(c), a["slots"], a["n"], a["K"], 256, 128, a["V"], 256, 128, a["dtype"], None)

    for fn in (append, read):
        assert fn(None) == qe.QE_ERR_INVALID_ARG
        for bad in BAD_CACHES:
            assert fn(_cache(**bad)) == qe.QE_ERR_INVALID_ARG, bad
        assert fn(_cache(group_size=16)) == qe.QE_ERR_UNSUPPORTED
        for bad in (dict(slots=None), dict(slots=0x1004), dict(n=-1), dict(dtype=3), dict(dtype=-1), dict(K=0x1001),
                    dict(dtype=qe.QE_F32, V=0x1002), dict(n=1 << 40)):
            assert fn(_cache(), **bad) == qe.QE_ERR_INVALID_ARG, bad
        assert fn(_cache(), n=0, K=None, V=None, slots=None) == qe.QE_OK     # nothing to do
    assert append(_cache(), K=None) == qe.QE_ERR_INVALID_ARG and append(_cache(), V=None) == qe.QE_ERR_INVALID_ARG
    assert read(_cache(), K=None, V=None) == qe.QE_ERR_INVALID_ARG


def _attention(**kw):
    f = dict(seqs=3, rows=3, q_heads=8, causal=1, window=0, scale=0.0, max_q=1, max_kv=100, q_start=_fake(1), kv_len=_fake(2),
             page_table=_fake(3), table_ld=2)
    f.update(kw)
    return qe.QEAttention(*[f[n] for n, _ in qe.QEAttention._fields_])


def test_attention_refuses(lib):
    def call(cache=None, Q=_fake(4), out=_fake(5), dtype=qe.QE_BF16, lse=None, ws=0x100000, ws_bytes=1 << 30, **kw):
        at = _attention(**kw)
        c = _cache(**(cache or {}))
        return lib.qe_cache_attention(ctypes.addressof(c), ctypes.addressof(at), Q, 1024, 128, out, 1024, 128, dtype, lse,
                                      ws, ws_bytes, None)

    for bad in BAD_CACHES:
        assert call(cache=bad) == qe.QE_ERR_INVALID_ARG, bad
    for bad in (dict(seqs=0), dict(seqs=65536), dict(rows=-1), dict(rows=1 << 31), dict(q_heads=0), dict(q_heads=7), dict(max_q=-1),
                dict(max_q=4), dict(max_kv=-1), dict(max_kv=(1 << 30) + 1), dict(window=-1), dict(window=5, causal=0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_start=None), dict(kv_len=None),
                dict(page_table=None), dict(table_ld=0), dict(table_ld=1 << 40), dict(q_start=0x1002), dict(Q=None),
                dict(out=None), dict(Q=0x1001), dict(out=0x1003), dict(lse=0x1002), dict(ws=0x100010), dict(dtype=7)):
        assert call(**bad) == qe.QE_ERR_INVALID_ARG, bad
    assert call(dtype=qe.QE_F32) == qe.QE_ERR_UNSUPPORTED
    assert call(rows=0, max_q=0, Q=None, out=None) == qe.QE_OK               # nothing to do
    c = _cache()
    assert lib.qe_cache_attention(ctypes.addressof(c), None, _fake(4), 1024, 128, _fake(5), 1024, 128, qe.QE_BF16, None, None,
                                  0, None) == qe.QE_ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    at = _attention()
    assert lib.qe_cache_attention_workspace(ctypes.addressof(c), ctypes.addressof(at), None) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_cache_attention_workspace(None, ctypes.addressof(at), ctypes.byref(n)) == qe.QE_ERR_INVALID_ARG
    at = _attention(q_heads=7)
    assert lib.qe_cache_attention_workspace(ctypes.addressof(c), ctypes.addressof(at), ctypes.byref(n)) == qe.QE_ERR_INVALID_ARG


def test_other_entry_points_take_no_fp16(lib):
    assert lib.qe_build_sigma(_fake(), qe.QE_F16, qe.QE_FEATURE_MAJOR, 8, 8, 8, _fake(2), 0, None) == qe.QE_ERR_INVALID_ARG
    assert lib.qe_quantize_layer(_fake(), qe.QE_F16, 4, 4, 4, _fake(2), 4, 1, None, _fake(3), _fake(4), _fake(5), _fake(6),
                                 None) == qe.QE_ERR_INVALID_ARG
