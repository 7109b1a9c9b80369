"""Attention behind a shared prefix: the workspace that is asked for does for every smaller batch too, and each device has its
limits raised.  The launches go to a runtime that runs none."""
import ctypes
import random

import pytest

from paper_2309_01885_gb300 import qe
from tests import cache_host as host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    lib = host.load(tmp_path_factory.mktemp("host"))
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    lib.qe_cache_attention_shared_workspace.argtypes = [vp, vp, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.qe_cache_attention_shared.argtypes = [vp, vp, vp, i64, vp, i64, i64, vp, i64, i64, ctypes.c_int, vp, vp, ctypes.c_size_t, vp]
    return lib


def workspace(lib, c, at, prefix):
    n = ctypes.c_size_t(0)
    assert lib.qe_cache_attention_shared_workspace(ctypes.addressof(c), ctypes.addressof(at), prefix, ctypes.byref(n)) == qe.QE_OK
    return n.value


def attend(lib, c, at, prefix, ws=None, ws_bytes=0, dtype=qe.QE_BF16):
    return lib.qe_cache_attention_shared(ctypes.addressof(c), ctypes.addressof(at), 0x9000, prefix, 0x4000, 128 * at.q_heads, 128, 0x5000,
                                         128 * at.q_heads, 128, dtype, None, ws, ws_bytes, None)


@pytest.mark.parametrize("seed", range(40))
def test_enough_for_every_smaller_batch(lib, seed):
    rng = random.Random(seed)
    kv_heads = rng.choice((1, 2, 3, 8, 32, 200))
    dim, group = rng.choice(((64, 32), (64, 64), (80, 32), (96, 32), (128, 32), (128, 128)))
    q_heads = kv_heads * rng.choice((1, 1, 4, 7, 29, 71))
    c = host.cache(kv_heads, dim, group)

    def up_to(n):
        return int(round(n ** rng.random())) if n else 0

    for _ in range(50):
        seqs, q, kv = up_to(300), up_to(4000), up_to(200000)
        rows, prefix = q + up_to(4000), up_to(kv)
        most = workspace(lib, c, host.batch(seqs, q, kv, q_heads, rows=rows), prefix)
        for _ in range(20):
            s, n, m, p = up_to(seqs), up_to(q), up_to(kv), up_to(prefix)
            at = host.batch(s, n, m, q_heads, rows=max(n, up_to(rows)))
            assert workspace(lib, c, at, p) <= most, (seqs, q, kv, rows, prefix, s, n, m, at.rows, p)
            assert attend(lib, c, at, p, 0x100000, most) == qe.QE_OK, (seqs, q, kv, rows, prefix, s, n, m, at.rows, p)


def test_every_device_has_its_limits_raised(lib):
    seen = []
    for device in (0, 1, 0):
        lib.fake_device(device, 152)
        for kv_heads, dim, group in ((8, 64, 32), (8, 64, 64), (8, 96, 32), (8, 128, 32), (8, 128, 64), (8, 128, 128)):
            for seqs, q, kv in ((1, 1, 500), (40, 1, 800), (64, 1, 30000), (2, 1, 100000), (64, 6, 9000), (1, 100, 5000), (30, 500, 3000)):
                for dtype in (qe.QE_BF16, qe.QE_F16):
                    before = lib.fake_launches()
                    assert attend(lib, host.cache(kv_heads, dim, group), host.batch(seqs, q, kv, 32), kv // 2, dtype=dtype) == qe.QE_OK
                    seen.append(lib.fake_launches() - before)
    lib.fake_device(0, 152)
    assert min(seen) >= 2                                # the prefix's pass and the one behind it
