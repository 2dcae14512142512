"""Where the bindings take the memory of a call on a given stream from (no GPU: torch's
streams are stand-ins, and no call is launched).  Outputs, their clearing and
workspaces that the binding allocates belong to the call's stream, since nothing orders
what the current stream has queued before that; outputs are kept for the current
stream too."""
import contextlib

import pytest
import torch

import paper_2405_11143_amd as pda
from paper_2405_11143_amd import pda as P

CURRENT, SIDE, OTHER = 11, 22, 33


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream = handle


def external_stream(handle, device=None):
    return Stream(handle or OTHER)  # (torch makes a new stream of a handle of 0)


class Recorder:
    """The stream that was current at each allocation and clearing, and the streams each tensor was kept for."""

    def __init__(self, monkeypatch):
        self.stack, self.made, self.cleared, self.kept = [CURRENT], {}, {}, {}
        empty, zero_ = torch.empty, torch.Tensor.zero_

        def recorded_empty(*args, **kw):
            t = empty(*args, **kw)
            self.made[id(t)] = (self.stack[-1], t)  # (kept alive: an id is one tensor's)
            return t

        def recorded_zero(t):
            self.cleared[id(t)] = self.stack[-1]
            return zero_(t)

        @contextlib.contextmanager
        def stream_context(stream):
            self.stack.append(stream.cuda_stream)
            yield
            self.stack.pop()

        monkeypatch.setattr(torch, "empty", recorded_empty)
        monkeypatch.setattr(torch.Tensor, "zero_", recorded_zero)
        monkeypatch.setattr(torch.Tensor, "record_stream",
                            lambda t, s: self.kept.setdefault(id(t), set()).add(s.cuda_stream))
        monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
        monkeypatch.setattr(torch.cuda, "stream", stream_context)
        monkeypatch.setattr(torch.cuda, "ExternalStream", external_stream)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(self.stack[-1]))
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(P.BoundCall, "__call__", lambda call: call.result)

    def check(self, outputs, cleared):
        for t in outputs:
            assert self.made[id(t)][0] == SIDE, "an output in the current stream's memory"
            assert CURRENT in self.kept[id(t)], "an output not kept for the stream it is handed to"
            if cleared:
                assert self.cleared[id(t)] == SIDE
        assert all(s == SIDE for s, _ in self.made.values()), "memory of the current stream"


@pytest.fixture(params=["stream", "handle"])
def given(request):
    return Stream(SIDE) if request.param == "stream" else SIDE


bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)


def fp8_inputs():
    cache = pda.make_fp8_cache(8, 2, 64, device="cpu")
    return cache, torch.zeros(3, 4, **i32), torch.zeros(3, **i32)


@pytest.mark.parametrize("name", ["bind_rotary_apply", "pda_rotary_apply"])
def test_rotary(monkeypatch, given, name):
    q, k, pos = torch.zeros(5, 4, 64, **bf), torch.zeros(5, 2, 64, **bf), torch.zeros(5, **i32)
    freq = torch.ones(32, dtype=torch.float64)
    rec = Recorder(monkeypatch)
    got = getattr(pda, name)(q, pos, pda.make_rotary(freq), k=k, stream=given)
    rec.check(got.result if name.startswith("bind") else got, cleared=True)


@pytest.mark.parametrize("name", ["bind_append_kv_fp8", "pda_append_kv_fp8"])
def test_append(monkeypatch, given, name):
    cache, table, lens = fp8_inputs()
    new, q = torch.zeros(3, 2, 2, 64, **bf), torch.zeros(3, 2, 4, 64, **bf)
    freq = torch.ones(32, dtype=torch.float64)
    rec = Recorder(monkeypatch)
    got = getattr(pda, name)(new, new, table, lens, *cache, max_context_len=64, rotary=pda.make_rotary(freq), q=q, stream=given)
    rec.check([got.result if name.startswith("bind") else got], cleared=True)


@pytest.mark.parametrize("name", ["bind_decode_fp8", "pda_decode_fp8"])
def test_decode(monkeypatch, given, name):
    cache, table, lens = fp8_inputs()
    q = torch.zeros(3, 2, 4, 64, **bf)
    rec = Recorder(monkeypatch)
    got = getattr(pda, name)(q, *cache, table, lens, 0.125, max_context_len=64, partition_tokens=16, stream=given)
    rec.check([got.result if name.startswith("bind") else got], cleared=False)
    assert len(rec.made) == 2  # the output and the workspace


def test_without_a_stream_nothing_changes_it(monkeypatch):
    cache, table, lens = fp8_inputs()
    q = torch.zeros(3, 2, 4, 64, **bf)
    rec = Recorder(monkeypatch)
    pda.pda_decode_fp8(q, *cache, table, lens, 0.125, max_context_len=64, partition_tokens=16)
    assert [s for s, _ in rec.made.values()] == [CURRENT] * 2 and not rec.kept


def test_the_null_stream_by_its_handle(monkeypatch):
    """0 is the default stream's handle: what the binding clears for a call on it is cleared there."""
    q, pos = torch.zeros(5, 4, 64, **bf), torch.zeros(5, **i32)
    rec = Recorder(monkeypatch)
    call = pda.bind_rotary_apply(q, pos, pda.make_rotary(torch.ones(32, dtype=torch.float64)), stream=0)
    assert call._args[-1].value is None  # (ctypes' null)
    out, _ = call.result
    assert rec.made[id(out)][0] == 0 and rec.cleared[id(out)] == 0
