"""What the cache's entry points allocate for a call on another stream belongs to that stream: memory that the current
stream has given back may still be in use there.  The library is a recorder, streams are names."""
import pytest
import torch

from paper_2309_01885_gb300 import qe
from tests.test_cache_python import Recorder, cache


@pytest.fixture
def made(monkeypatch):
    """(function, stream that was current) of every allocation; the stream of every call to the library."""
    now, made, rec = ["current"], [], Recorder()

    class Stream:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.was = now[0]
            if self.stream is not None:
                now[0] = self.stream.cuda_stream

        def __exit__(self, *a):
            now[0] = self.was

    empty, contiguous = torch.empty, torch.Tensor.contiguous
    monkeypatch.setattr(qe, "_lib", rec)
    monkeypatch.setattr(qe, "_raw_stream", lambda index: now[0])
    monkeypatch.setattr(torch.cuda, "stream", Stream)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(("empty", now[0])) or empty(*a, **k))
    monkeypatch.setattr(torch.Tensor, "contiguous", lambda t: made.append(("contiguous", now[0])) or contiguous(t))
    return made, rec


class Other:
    cuda_stream = "other"


@pytest.mark.parametrize("stream,name", [(None, "current"), (Other(), "other")])
def test_results_are_allocated_on_the_calls_stream(made, stream, name):
    made, rec = made
    c, slots = cache(), torch.arange(3)
    k, v = qe.qe_cache_read(c, slots, stream=stream)
    assert made == [("empty", name)] * 2 and rec.calls[-1]["args"][-1] == name
    made.clear()
    table = torch.zeros(3, 9, dtype=torch.int32)[:, 2:5]
    args = (torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.arange(4, dtype=torch.int32), torch.ones(3, dtype=torch.int32), table, 1, 40)
    out = qe.qe_cache_attention(c, *args, stream=stream)
    assert sorted(made) == [("contiguous", name), ("empty", name)] and rec.calls[-1]["args"][-1] == name
    # with results of the caller's nothing is allocated
    made.clear()
    qe.qe_cache_read(c, slots, k=k, v=v, stream=stream)
    assert qe.qe_cache_attention(c, *args[:3], table.clone(), 1, 40, out=out, stream=stream) is out and made == []
    qe.qe_cache_append(c, torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), slots, stream=stream)
    assert rec.calls[-1]["args"][-1] == name
