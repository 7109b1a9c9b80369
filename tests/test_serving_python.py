"""The serving operators' Python entry points without a GPU: device, stream and allocations of each call.  The library is a
recorder, tensors say that they are on the device that a test names."""
import pytest
import torch

from paper_2309_01885_gb300 import qe
from tests.test_cache_python import Recorder, cache


class Switch:
    """torch.cuda.device or torch.cuda.stream: what is current while a call runs."""

    def __init__(self, now, key, value):
        self.now, self.key, self.value = now, key, value

    def __enter__(self):
        self.was = self.now[self.key]
        if self.value is not None:
            self.now[self.key] = self.value

    def __exit__(self, *a):
        self.now[self.key] = self.was


@pytest.fixture
def world(monkeypatch):
    """What is current; calls as (name, device, stream); allocations as (device, stream)."""
    now, calls, made = dict(device=0, stream="current"), [], []
    rec, plain, empty = Recorder(), Recorder.__getattr__, torch.empty

    def note(self, name):
        call = plain(self, name)
        return lambda *args: calls.append((name, now["device"], now["stream"])) or call(*args)

    monkeypatch.setattr(Recorder, "__getattr__", note)
    monkeypatch.setattr(qe, "_lib", rec)
    monkeypatch.setattr(qe, "_raw_stream", lambda index: now["stream"])
    monkeypatch.setattr(qe, "_current_device", lambda: now["device"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: Switch(now, "device", d))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: Switch(now, "stream", getattr(s, "cuda_stream", None)))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 5)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append((now["device"], now["stream"])) or empty(*a, **k))
    return now, calls, made, rec


class Other:
    cuda_stream = "other"


def integers(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def operators():
    c = cache()
    c._index = 5
    pool = qe.PagePool(c)
    w = object.__new__(qe.QuantizedWeights)
    w.q, w.p, w.bits, w.group_size, w.device, w._ref, w._index = 96, 64, 4, 0, torch.device("cpu"), 0, 5
    x, heads = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    rope = qe.Rope(64)
    return dict(
        qe_cache_grow=(lambda **k: qe.qe_cache_grow(c, pool, integers(3), integers(3), integers(3, 4), 8, **k), 3),
        qe_norm_rotate=(lambda **k: qe.qe_norm_rotate(heads, heads[:, :2], integers(3), rope, **k), 2),
        qe_linear=(lambda **k: qe.qe_linear(w, x, **k), 1),
        qe_cache_attention_shared=(lambda **k: qe.qe_cache_attention_shared(c, heads, integers(4), integers(3), integers(3, 4), 1, 40,
                                                                             integers(2), 20, **k), 1))


@pytest.mark.parametrize("name", ["qe_cache_grow", "qe_norm_rotate", "qe_linear", "qe_cache_attention_shared"])
@pytest.mark.parametrize("current", [0, 5])
@pytest.mark.parametrize("stream,called", [(None, "current"), (Other(), "other")])
def test_calls_go_to_their_device_and_stream(world, name, current, stream, called):
    now, calls, made, _ = world
    call, results = operators()[name]
    calls.clear(), made.clear()
    now["device"] = current
    call(stream=stream)
    (got, device, on), = calls
    # (a stream that is given is of its device: what torch.cuda.stream makes current)
    assert got == name and on == called and (device == 5 or stream is not None)
    assert made == [(device, called)] * results
    assert now == dict(device=current, stream="current")


def test_results_of_the_callers_are_not_allocated(world):
    _, calls, made, rec = world
    ops = operators()
    q_start, slots, positions = integers(4), torch.zeros(8, dtype=torch.int64), integers(8)
    q, k, y = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 96, dtype=torch.bfloat16)
    made.clear()
    assert all(a is b for a, b in zip(ops["qe_cache_grow"][0](q_start=q_start, slots=slots, positions=positions), (q_start, slots, positions)))
    assert all(a is b for a, b in zip(ops["qe_norm_rotate"][0](q_out=q, k_out=k), (q, k)))
    assert ops["qe_linear"][0](out=y) is y and ops["qe_cache_attention_shared"][0](out=q) is q
    assert made == [] and [c[0] for c in calls if c[0] != "qe_rope_init"] == list(ops)


def test_what_the_library_is_given(world):
    """Addresses, pitches and counts of strided tensors."""
    _, _, _, rec = world
    fused = torch.zeros(3, 8, 64, dtype=torch.float16)
    q, k = fused[:, :4], fused[:, 4:6]
    weight = torch.ones(64, dtype=torch.bfloat16)
    qe.qe_norm_rotate(q, k, None, None, k_weight=weight, eps=0.5, q_out=q, k_out=k)
    got = qe.QEHeads.from_buffer_copy(rec.calls[-1]["args"][0] + b"\0" * 8)
    want = dict(tokens=3, q_heads=4, k_heads=2, head_dim=64, dtype=qe.QE_F16, weight_dtype=qe.QE_BF16, eps=0.5)
    assert {n: getattr(got, n) for n in want} == want
    assert [v for n, v in ((n, getattr(got, n)) for n, _ in got._fields_) if v == fused.data_ptr()] == [fused.data_ptr()] * 2
    x = torch.zeros(3, 100, dtype=torch.bfloat16)[:, 10:74]
    w = object.__new__(qe.QuantizedWeights)
    w.q, w.p, w.bits, w.group_size, w.device, w._ref, w._index = 96, 64, 4, 0, torch.device("cpu"), 0, 5
    qe.qe_linear(w, x, activation="silu")
    got = qe.QEProduct.from_buffer_copy(rec.calls[-1]["args"][1] + b"\0" * 8)
    assert (got.rows, got.X, got.ldx, got.ldy, got.bias, got.residual, got.act) == (3, x.data_ptr(), 100, 96, None, None, qe.ACTIVATIONS["silu"])
    for bad in (x[:, :63], x.t(), x[0]):
        with pytest.raises((ValueError, TypeError)):
            qe.qe_linear(w, bad)


def test_shared_refuses_too_few_prefix_pages(world):
    c = cache()
    c._index = 5
    with pytest.raises(ValueError):
        qe.qe_cache_attention_shared(c, torch.zeros(3, 4, 64, dtype=torch.bfloat16), integers(4), integers(3), integers(3, 4), 1, 40,
                                     integers(2), 33)
