"""Calls on a given stream while the current stream still has work queued on memory that
it has freed: neither sees the other's bytes."""
import numpy as np
import pytest
import torch

import paper_2405_11143_amd as pda
import workloads as W
from test_gpu_fp8 import case, dev, up, upload  # noqa: F401

pytestmark = pytest.mark.gpu


def behind_pending_work(dev, sizes, call, want):  # noqa: F811
    """Runs `call` on a stream of its own while tensors of the given sizes (bytes), already freed, wait to be written
    and read on the current stream."""
    busy = torch.randn(4096, 4096, device=dev, dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):  # (a stream, or its handle)
        torch.cuda.synchronize()
        freed = [torch.zeros(n, dtype=torch.uint8, device=dev) for n in sizes for _ in range(2)]
        for _ in range(40):
            busy = (busy @ busy).clamp_(-1, 1)
        sums = []
        for i, t in enumerate(freed):
            t.fill_(i + 1)
        for _ in range(20):
            busy = (busy @ busy).clamp_(-1, 1)
        for t in freed:
            sums.append(t.to(torch.int32))
        del freed, t
        got = call(stream)
        torch.cuda.synchronize()
        for i, s in enumerate(sums):
            assert (s == i + 1).all(), "the call wrote to memory that was still in use"
        got, ref = (x if isinstance(x, tuple) else (x,) for x in (got, want))
        for a, b in zip(got, ref):
            assert torch.equal(a, b), "work of the current stream reached the call's results"


def test_rotary_and_append(dev):  # noqa: F811
    st, cache, q, K, V = case([300, 77, 2], 8, 2, 128, 3, 32, dev)
    rot = pda.make_rotary(up(pda.pda_rotary_inv_freq(128)[0], dev))
    rows, keys = q.reshape(9, 8, 128), up(np.random.RandomState(5).randn(9, 2, 128), dev, torch.bfloat16)
    positions = up(np.array([0, 5, 3, -1, 7, 8, 1000, -2, 4], np.int32), dev)
    sizes = [rows.numel() * 2, keys.numel() * 2]
    behind_pending_work(dev, sizes, lambda s: pda.pda_rotary_apply(rows, positions, rot, k=keys, stream=s),
                        pda.pda_rotary_apply(rows, positions, rot, k=keys))
    new, table, lens = keys.reshape(3, 3, 2, 128), up(st.block_table, dev), up(st.context_lens, dev)
    on_gpu = upload(cache, dev)
    call = lambda **kw: pda.pda_append_kv_fp8(new, new, table, lens, *on_gpu, max_context_len=st.max_context_len, rotary=rot,
                                              q=q, **kw)
    behind_pending_work(dev, [q.numel() * 2], lambda s: call(stream=s), call())


@pytest.mark.parametrize("n", [1, 5, 30])
def test_attention_over_the_8_bit_cache(dev, n):  # noqa: F811
    st, cache, q, K, V = case([300, 77, 1, 250] * 10, 8, 2, 128, n, 31, dev)
    on_gpu, table, lens = upload(cache, dev), up(st.block_table, dev), up(st.context_lens, dev)
    kw = dict(max_context_len=st.max_context_len, partition_tokens=48)
    need = pda.pda_plan_fp8(pda.make_problem(len(st.context_lens), 8, 2, 128, st.num_blocks, table.shape[1],
                                             st.max_context_len, 48, num_query_tokens=n))["workspace_bytes"]
    call = lambda **more: pda.pda_decode_fp8(q, *on_gpu, table, lens, st.scale, **kw, **more)
    behind_pending_work(dev, [q.numel() * 4, need], lambda s: call(stream=s), call())


@pytest.mark.parametrize("n", [1, 5])
def test_attention_over_the_bf16_cache(dev, n):  # noqa: F811
    st, cache, q, K, V = case([300, 77, 1, 250] * 10, 8, 2, 128, n, 31, dev)
    k = W.k_rows_to_cache(up(K, dev, torch.bfloat16))
    v, table, lens = up(V, dev, torch.bfloat16), up(st.block_table, dev), up(st.context_lens, dev)
    prob = pda.make_problem(len(st.context_lens), 8, 2, 128, st.num_blocks, table.shape[1], st.max_context_len, 48,
                            num_query_tokens=n)
    call = lambda **more: pda.pda_decode(q, k, v, table, lens, st.scale, max_context_len=st.max_context_len,
                                         partition_tokens=48, **more)
    behind_pending_work(dev, [q.numel() * 4, pda.pda_workspace_bytes(prob)], lambda s: call(stream=s), call())


def test_logprobs(dev):  # noqa: F811
    logits, tokens = torch.randn(33, 40000, device=dev), torch.arange(33, dtype=torch.int32, device=dev)
    call = lambda **more: pda.pda_token_logprobs(logits, tokens, **more)
    behind_pending_work(dev, [33 * 4, 33 * 4, pda.pda.pda_logprob_workspace_bytes(33, 40000, 1)], lambda s: call(stream=s), call())


@pytest.mark.parametrize("model", [False, True])
def test_captured_graphs(dev, model):  # noqa: F811
    """A graph made behind pending work, whose class allocates the workspace (and the output), launched on another stream
    at once."""
    st, cache, q, K, V = case([300, 77, 1, 250] * 10, 8, 2, 128, 1, 31, dev)
    k, v = W.k_rows_to_cache(up(K, dev, torch.bfloat16)), up(V, dev, torch.bfloat16)
    table, lens = up(st.block_table, dev), up(st.context_lens, dev)
    new = torch.randn(len(st.context_lens), 1, 2, 128, device=dev).to(torch.bfloat16)
    kw = dict(max_context_len=st.max_context_len, partition_tokens=48)
    pda.pda_append_kv(new, new, table, lens, k, v, max_context_len=st.max_context_len)
    want = pda.pda_decode(q, k, v, table, lens, st.scale, **kw)
    need = pda.pda_workspace_bytes(pda.make_problem(len(st.context_lens), 8, 2, 128, st.num_blocks, table.shape[1],
                                                    st.max_context_len, 48))

    def call(stream):
        if model:
            out = torch.zeros_like(want)
            torch.cuda.synchronize()
            graph = pda.ModelStepGraph([dict(q=q, k_new=new, v_new=new, k_cache=k, v_cache=v, out=out)], table, lens, st.scale,
                                       **kw)
            graph.launch(stream)
        else:
            graph = pda.StepGraph(q, new, new, k, v, table, lens, st.scale, **kw)
            out = graph.launch(stream)
        torch.cuda.synchronize()
        return out

    behind_pending_work(dev, [q.numel() * 4, need], call, want)
