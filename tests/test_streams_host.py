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


def bf16_inputs(n=1):
    q = torch.zeros(3, n, 4, 64, **bf)
    return q, torch.zeros(8, 2, 8, 16, 8, **bf), torch.zeros(8, 2, 16, 64, **bf), torch.zeros(3, 4, **i32), torch.zeros(3, **i32)


@pytest.mark.parametrize("name", ["bind_decode", "pda_decode", "pda_partition_attention", "bind_decode_append",
                                  "pda_decode_append", "bind_decode_noalloc", "pda_decode_noalloc"])
def test_bf16_step(monkeypatch, given, name):
    q, k, v, table, lens = bf16_inputs()
    new = torch.zeros(3, 1, 2, 64, **bf)
    rec = Recorder(monkeypatch)
    args = (q, new, new, k, v) if "append" in name else (q, k, v)
    got = getattr(pda, name)(*args, table, lens, 0.125, max_context_len=64, partition_tokens=16, stream=given)
    rec.check([got.result if name.startswith("bind") else got], cleared=False)
    assert len(rec.made) == (1 if "noalloc" in name else 2)


def test_bf16_shared_prefix(monkeypatch, given):
    q, k, v, table, lens = bf16_inputs()
    start, prefix = torch.tensor([0, 2], **i32), torch.tensor([16], **i32)
    lib = pda.load_library()

    class Library:  # (this one is not a bound call)
        def __getattr__(self, name):
            return (lambda *args: P.PDA_OK) if name == "pda_decode_shared_prefix" else getattr(lib, name)

    rec = Recorder(monkeypatch)
    monkeypatch.setattr(P, "load_library", Library)
    out = pda.pda_decode_shared_prefix(q, k, v, table, lens, 0.125, start, prefix, max_context_len=64, max_group_size=2,
                                       max_prefix_len=16, stream=given)
    rec.check([out], cleared=False)
    assert len(rec.made) == 2


@pytest.mark.parametrize("name", ["bind_token_logprobs", "pda_token_logprobs"])
def test_logprobs(monkeypatch, given, name):
    logits, tokens = torch.zeros(5, 128256), torch.zeros(5, **i32)
    rec = Recorder(monkeypatch)
    got = getattr(pda, name)(logits, tokens, stream=given)
    rec.check(got.result if name.startswith("bind") else got, cleared=False)
    assert len(rec.made) == 3


def test_ceilings(monkeypatch, given):
    q, k, v, table, lens = bf16_inputs()
    rec = Recorder(monkeypatch)
    for call in (pda.bind_gather_ceiling(torch.zeros(4, **i32), k, v, 8, stream=given),
                 pda.bind_stream_ceiling(k, 8, stream=given)):
        rec.check([call.result], cleared=False)


@pytest.mark.parametrize("model", [False, True])
def test_graphs(monkeypatch, given, model):
    """What a captured graph's class allocates is idle when the graph is made, and kept for every stream it is
    launched on; tensors that are given are left alone."""
    q, k, v, table, lens = bf16_inputs()
    new = torch.zeros(3, 1, 2, 64, **bf)
    lib = pda.load_library()

    class Library:
        def __getattr__(self, name):
            return (lambda *args: P.PDA_OK) if "graph" in name else getattr(lib, name)

    rec = Recorder(monkeypatch)
    monkeypatch.setattr(P, "load_library", Library)
    waits = []
    monkeypatch.setattr(Stream, "synchronize", lambda s: waits.append(s.cuda_stream), raising=False)

    def make(**kw):
        if not model:
            return pda.StepGraph(q, new, new, k, v, table, lens, 0.125, max_context_len=64, partition_tokens=16, **kw)
        layer = dict(q=q, k_new=new, v_new=new, k_cache=k, v_cache=v, out=torch.zeros(3, 1, 4, 64))
        kw.pop("out", None)
        return pda.ModelStepGraph([layer], table, lens, 0.125, max_context_len=64, partition_tokens=16, **kw)

    graph = make()
    made = [graph.workspace] + ([] if model else [graph.out])
    assert waits == [CURRENT] and {id(t) for t in made} == set(rec.made)
    graph.launch(given)
    graph.launch(given)
    assert all(rec.kept[id(t)] == {SIDE} for t in made)
    graph.launch()
    assert all(rec.kept[id(t)] == {SIDE, CURRENT} for t in made)
    rec.kept.clear()
    mine = make(workspace=graph.workspace, out=torch.zeros(3, 1, 4, 64))
    mine.launch(given)
    assert waits == [CURRENT] and not rec.kept


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
