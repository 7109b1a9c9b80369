"""The cache's host code over a CUDA runtime that launches nothing (tests/fake_cudart.cpp)."""
import ctypes
import os
import subprocess

from paper_2309_01885_gb300 import build, qe

OBJECTS = ["qe_cache.o", "qe_attend.o", "qe_attend_whole8.o", "qe_attend_whole4.o", "qe_attend_tc.o"]


def load(folder):
    """A copy of its own, so that nothing that an earlier test left behind is kept."""
    build.build_lib()
    objs = [os.path.join(build.OUT_DIR, o) for o in OBJECTS]
    if not all(os.path.exists(o) for o in objs):
        build.build_lib(force=True)
    out = os.path.join(str(folder), "libqe_host.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "fake_cudart.cpp")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", f"-I{cuda}", "-o", out, src, *objs])
    lib = ctypes.CDLL(out)
    lib.fake_kernel.restype = ctypes.c_char_p
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    lib.qe_cache_attention_workspace.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_size_t)]
    lib.qe_cache_attention.argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, ctypes.c_int, vp, vp, ctypes.c_size_t, vp]
    return lib


def cache(kv_heads=8, dim=128, group=32, page=64):
    return qe.QECache(0x100000, 1 << 50, 1 << 20, page, kv_heads, dim, group)


def batch(seqs, max_q, max_kv, q_heads, window=0, causal=1, rows=None):
    return qe.QEAttention(seqs, seqs * max_q if rows is None else rows, q_heads, causal, window, 0.0, max_q, max_kv, 0x1000, 0x2000,
                          0x3000, 1 << 10)


def workspace(lib, c, at):
    n = ctypes.c_size_t(0)
    assert lib.qe_cache_attention_workspace(ctypes.addressof(c), ctypes.addressof(at), ctypes.byref(n)) == qe.QE_OK
    return n.value


def attend(lib, c, at, ws=None, ws_bytes=0, dtype=qe.QE_BF16):
    return lib.qe_cache_attention(ctypes.addressof(c), ctypes.addressof(at), 0x4000, 128 * at.q_heads, 128, 0x5000, 128 * at.q_heads, 128,
                                  dtype, None, ws, ws_bytes, None)
