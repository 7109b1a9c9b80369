"""Attention over the 4-bit cache on more than one device of a process, its launches going to a runtime that runs none."""
import pytest
import torch

from paper_2309_01885_gb300 import qe
from tests import cache_host as host
from tests.test_cache_python import Recorder, cache

# every form of the kernels: (seqs, query rows, longest context), at 1, 2 and 4 row tiles, whole items and dealt out, tiles
CALLS = [(1, 1, 500), (3, 1, 500), (40, 1, 800), (40, 2, 800), (40, 3, 800), (2, 1, 100000), (2, 3, 100000), (64, 6, 9000),
         (1, 100, 5000), (30, 500, 3000)]
CACHES = [(8, 64, 32), (8, 64, 64), (8, 96, 32), (8, 128, 32), (8, 128, 64), (8, 128, 128)]


@pytest.fixture
def lib(tmp_path):
    return host.load(tmp_path)


def run_all(lib):
    seen = set()
    for kv_heads, dim, group in CACHES:
        for seqs, q, kv in CALLS:
            for dtype in (qe.QE_BF16, qe.QE_F16):
                for q_heads in (8, 32):
                    before = lib.fake_launches()
                    assert host.attend(lib, host.cache(kv_heads, dim, group), host.batch(seqs, q, kv, q_heads), dtype=dtype) == qe.QE_OK, \
                        (dim, group, seqs, q, kv, lib.fake_kernel())
                    assert lib.fake_launches() > before
                    seen.add(lib.fake_kernel())
    return seen


def test_every_device_has_its_limits_raised(lib):
    lib.fake_device(0, 152)
    first = run_all(lib)
    lib.fake_device(1, 152)
    assert run_all(lib) == first and len(first) > 30
    lib.fake_device(0, 152)
    run_all(lib)


def test_a_limit_that_was_refused_is_asked_for_again(lib):
    c, at = host.cache(), host.batch(1, 100, 5000, 32)
    lib.fake_fail_attribute(1)
    assert host.attend(lib, c, at) == qe.QE_ERR_CUDA
    assert host.attend(lib, c, at) == qe.QE_OK


def test_work_is_dealt_out_over_the_current_device(lib):
    c, at = host.cache(), host.batch(64, 1, 100000, 32)
    grids = {}
    for d, sms in ((0, 152), (1, 76), (2, 148), (0, 152)):
        lib.fake_device(d, sms)
        assert host.attend(lib, c, at) == qe.QE_OK
        grids[sms] = lib.fake_grid(0)
    assert grids[152] == 2 * grids[76] and grids[152] // 152 == grids[148] // 148 and grids[152] % 152 == 0


# ---- the Python entry points ----

@pytest.fixture
def recorder(monkeypatch):
    """Tensors say that they are on device 5; device 0 is the current one."""
    rec, now = Recorder(), [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was, now[0] = now[0], self.index

        def __exit__(self, *a):
            now[0] = self.was

    seen = []
    plain = Recorder.__getattr__

    def note(self, name):
        call = plain(self, name)

        def wrapped(*args):
            seen.append((name, now[0]))
            return call(*args)
        return wrapped

    monkeypatch.setattr(Recorder, "__getattr__", note)
    monkeypatch.setattr(qe, "_lib", rec)
    monkeypatch.setattr(qe, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(qe, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 5)
    return seen, now


def test_entry_points_make_the_caches_device_current(recorder):
    seen, now = recorder
    c = cache()
    c._index = 5
    x, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.arange(3)
    qe.qe_cache_append(c, x, x, slots)
    qe.qe_cache_read(c, slots)
    qe.qe_cache_attention(c, torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.arange(4, dtype=torch.int32), torch.ones(3, dtype=torch.int32),
                          torch.zeros(3, 2, dtype=torch.int32), 1, 20)
    qe.qe_cache_attention_workspace(c, 3, 4, 3, 1, 40)
    assert seen == [(n, 5) for n in ("qe_cache_append", "qe_cache_read", "qe_cache_attention", "qe_cache_attention_workspace")]
    assert now == [0]
