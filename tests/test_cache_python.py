"""The cache's Python entry points without a GPU: what they hand to the library, which is a recorder here."""
import ctypes

import pytest
import torch

from paper_2309_01885_gb300 import qe


class Recorder:
    """Stands for the library: keeps each call's arguments (of attention also its qe_attention) and returns 0."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            note = dict(name=name, args=args)
            if name == "qe_cache_attention":
                note["at"] = {f: getattr(qe.QEAttention.from_address(args[1]), f) for f, _ in qe.QEAttention._fields_}
                ld, seqs = note["at"]["table_ld"], note["at"]["seqs"]
                note["table"] = list((ctypes.c_int32 * (ld * seqs)).from_address(note["at"]["page_table"])) if ld > 0 else []
            self.calls.append(note)
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(qe, "_lib", rec)
    monkeypatch.setattr(qe, "_raw_stream", lambda index: 0)
    return rec


def cache(pages=8, page_size=16, kv_heads=2, head_dim=64, group_size=32):
    """A cache on the CPU, as its entry points see one."""
    c = object.__new__(qe.KVCache)
    c.pages, c.page_size, c.kv_heads, c.head_dim, c.group_size = pages, page_size, kv_heads, head_dim, group_size
    c.device, c._ref, c._index = torch.device("cpu"), 0, -1
    return c


def attend(table, **kw):
    seqs = table.shape[0]
    return qe.qe_cache_attention(cache(), torch.zeros(seqs, 4, 64, dtype=torch.bfloat16), torch.arange(seqs + 1, dtype=torch.int32),
                                 torch.ones(seqs, dtype=torch.int32), table, 1, 40, **kw)


WIDE = torch.arange(5 * 12, dtype=torch.int32).view(5, 12)


@pytest.mark.parametrize("table", [
    WIDE, WIDE[:, 2:7], WIDE[:, :3], WIDE[:, 9:], WIDE[::2], WIDE[1:2, 3:8], WIDE[:1], WIDE.t(), WIDE.t()[:, :2], WIDE.t()[4:5],
    torch.zeros(5, 1, dtype=torch.int32).t(), WIDE[:1, :4].expand(3, 4), WIDE[:, :1]])
def test_page_table_as_the_library_takes_it(lib, table):
    """Whatever strides a table has, the library gets its rows one after the other, and their length as the limit."""
    attend(table)
    got, = lib.calls
    assert got["at"]["table_ld"] == table.shape[1] and got["at"]["seqs"] == table.shape[0]
    assert got["table"] == table.flatten().tolist()


def test_page_table_is_checked(lib):
    for bad in (WIDE.long(), WIDE[0], WIDE[None]):
        with pytest.raises(ValueError):
            qe.qe_cache_attention(cache(), torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.arange(6, dtype=torch.int32),
                                  torch.ones(5, dtype=torch.int32), bad, 1, 40)
    assert not lib.calls
