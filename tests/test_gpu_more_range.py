"""Head norms, windowed attention and block tables over the range of their sizes: every way that
tokens are shared out, more tokens than a launch has workgroups, offsets past 32 bits, long lists,
workspaces that captured graphs share, pools whose contents contradict themselves."""
import numpy as np
import pytest
import torch

import more_reference as ref
import paper_2405_11143_amd as pda
import test_gpu_norm_rotary as heads
import test_gpu_window as windows
from more_reference import cache_of

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


# --------------------------------------------------------------- head norms --

@pytest.mark.parametrize("T", [2047, 4097, 9001, 16383, 16385])
@pytest.mark.parametrize("Hq,Hkv,D,R", [(4, 1, 128, 128), (9, 2, 64, 32), (3, 0, 80, 80), (16, 2, 16, 16)])
def test_forward_of_many_tokens(T, Hq, Hkv, D, R):
    heads.test_forward((T, Hq, Hkv, D, R), BF, dict(axes=2, offset=1.0))
    heads.test_forward((T, Hq, Hkv, D, R), F32, dict(norm=False, interleaved=True))


@pytest.mark.parametrize("T", [4097, 16385])
@pytest.mark.parametrize("Hq,Hkv,D,R", [(4, 1, 128, 128), (9, 2, 64, 32), (3, 0, 80, 80)])
def test_backward_of_many_tokens(T, Hq, Hkv, D, R):
    heads.test_backward((T, Hq, Hkv, D, R), BF, dict(axes=2, offset=1.0))
    heads.test_backward((T, Hq, Hkv, D, R), F32, dict(interleaved=True))


@pytest.mark.parametrize("T", [4097, 16385])
@pytest.mark.parametrize("Hq,Hkv,D,R", [(4, 1, 128, 128), (9, 2, 64, 32)])
def test_append_of_many_tokens(T, Hq, Hkv, D, R):
    heads.test_append(T, Hq, Hkv, D, R, dict(axes=2, offset=1.0))


@pytest.mark.parametrize("Hq,Hkv,D,R", [(4, 1, 128, 128), (8, 2, 64, 32), (32, 8, 128, 128)])
def test_many_tokens_in_place(Hq, Hkv, D, R):
    """Wavefronts that loop over tokens, and ones that do not: over the rows themselves the same bits as beside them."""
    c = heads.Case(12001, Hq, Hkv, D, R)
    want = pda.pda_norm_rotary(c.q, c.pos_arg, c.k, **c.kw_args)
    rows = c.rows.clone()
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hkv]
    pda.pda_norm_rotary(q, c.pos_arg, k, q_out=q, k_out=k, **c.kw_args)
    assert torch.equal(q[c.real], want[0][c.real]) and torch.equal(k[c.real], want[1][c.real])
    assert torch.equal(rows[~c.real], c.rows[~c.real]) and torch.equal(rows[:, Hq + Hkv:], c.rows[:, Hq + Hkv:])


def test_more_tokens_than_workgroups():
    """2^20 workgroups of 4 tokens, and some."""
    c = heads.Case(4 * 2 ** 20 + 77, 1, 0, 16, 16)
    out, _ = pda.pda_norm_rotary(c.q, c.pos_arg, **c.kw_args)
    heads.assert_rows(out, *c.exact(c.q, c.qw), c.real)


def test_rows_past_32_bits():
    """Tokens 2.2 GB apart: both directions, and the keys and values on their way to the cache."""
    c = heads.Case(4, 3, 2, 64, 64, padding=False)

    def apart(t):
        far = torch.empty(3 * 1100000000 + t[0].numel(), dtype=BF, device="cuda").as_strided(t.shape, (1100000000, 64, 1))
        far.copy_(t)
        return far

    g, gk = torch.randn_like(c.q.contiguous()), torch.randn_like(c.k.contiguous())
    near = pda.pda_norm_rotary(c.q, c.pos_arg, c.k, **c.kw_args)
    near_grad = pda.pda_norm_rotary_backward(c.q, g, c.pos_arg, c.k, gk, **c.kw_args)
    q, k = apart(c.q), apart(c.k)
    q_out, k_out = apart(torch.zeros_like(g)), apart(torch.zeros_like(gk))
    pda.pda_norm_rotary(q, c.pos_arg, k, q_out=q_out, k_out=k_out, **c.kw_args)
    assert torch.equal(q_out, near[0]) and torch.equal(k_out, near[1])
    caches = [[torch.zeros(2, 2, 8, 16, 8, dtype=BF, device="cuda"), torch.zeros(2, 2, 16, 64, dtype=BF, device="cuda")]
              for _ in range(2)]
    slots = i32([3, 31, 16, 0])
    pda.pda_norm_rotary_append(c.q, c.k, c.v, c.pos_arg, slots, *caches[0], **c.kw_args)
    pda.pda_norm_rotary_append(q, k, apart(c.v), c.pos_arg, slots, *caches[1], q_out=q_out, **c.kw_args)
    assert torch.equal(q_out, near[0])
    for x, y in zip(*caches):
        assert torch.equal(x, y)
    pda.pda_norm_rotary_backward(q, apart(g), c.pos_arg, k, apart(gk), dq=q_out, dk=k_out, **c.kw_args)
    assert torch.equal(q_out, near_grad[0]) and torch.equal(k_out, near_grad[1])


def test_two_graphs_with_one_gradient_workspace():
    """Captured one after the other, replayed in turns."""
    cases = [heads.Case(T, 4, 2, 64, 64, seed=T) for T in (700, 90)]
    size = max(pda.pda_norm_rotary_workspace_bytes(c.T, 4, 2, 64) for c in cases)
    workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
    stream, graphs = torch.cuda.Stream(), []
    calls = [pda.bind_norm_rotary_backward(c.q, c.q, c.pos_arg, c.k, c.k, workspace=workspace, stream=stream, **c.kw_args)
             for c in cases]
    want = [[t.clone() for t in pda.pda_norm_rotary_backward(c.q, c.q, c.pos_arg, c.k, c.k, **c.kw_args)] for c in cases]
    torch.cuda.synchronize()
    for call in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call()
    for which in (0, 1, 0, 1, 1, 0):
        for t in calls[which].result:
            t.zero_()
        graphs[which].replay()
        torch.cuda.synchronize()
        for x, y in zip(calls[which].result, want[which]):
            assert torch.equal(x, y)


# ---------------------------------------------------------------- attention --

@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 1), (8, 2, 6), (16, 1, 9)])
def test_long_lists(Hq, Hkv, n):
    """More blocks to a work item than are held at once: 64 to a wavefront, 1024 to a workgroup."""
    q, k, v, table, lens = windows.setup(2, Hq, Hkv, 64, n, [17003, 40], n)
    windows.check(q, k, v, table, lens, 16900, 5, partition_tokens=17024)


@pytest.mark.parametrize("n", [1, 5, 40])
def test_cache_past_32_bits(n):
    """Blocks beyond 4 GiB of K and of V."""
    q, k, v, table, lens = windows.setup(2, 8, 8, 128, n, [200, 333], n)
    near = windows.run(q, k, v, table, lens, 150, 5)
    NB, held = 140000, k.shape[0]
    kc = torch.empty(NB, 8, 16, 16, 8, dtype=BF, device="cuda")
    vc = torch.empty(NB, 8, 16, 128, dtype=BF, device="cuda")
    place = np.arange(held) * ((NB - 1) // (held - 1))
    place[-1] = NB - 1
    at = torch.from_numpy(place).cuda()
    kc[at], vc[at] = (t.cuda() for t in cache_of(k, v))
    far = np.where(table >= 0, place[np.maximum(table, 0)], -1)
    qd = q.cuda() if n > 1 else q[:, 0].contiguous().cuda()
    got = pda.pda_decode_window(qd, kc, vc, i32(far), i32(lens), 128 ** -0.5, window=150, sinks=5,
                                max_context_len=16 * table.shape[1])
    assert torch.equal(got.view(near.shape), near)


def test_append_past_32_bits():
    c = heads.Case(6, 2, 8, 128, 128, padding=False)
    NB = 140000
    kc = torch.zeros(NB, 8, 16, 16, 8, dtype=BF, device="cuda")
    vc = torch.zeros(NB, 8, 16, 128, dtype=BF, device="cuda")
    slots = i32([16 * NB - 1, 16 * NB - 16, 16 * 135000 + 7, 16 * 70000 + 3, 0, 16 * NB])
    pda.pda_norm_rotary_append(c.q, c.k, c.v, c.pos_arg, slots, kc, vc, **c.kw_args)
    near_k = torch.zeros(1, 8, 16, 16, 8, dtype=BF, device="cuda")
    near_v = torch.zeros(1, 8, 16, 128, dtype=BF, device="cuda")
    pda.pda_norm_rotary_append(c.q, c.k, c.v, c.pos_arg, i32([0, 1, 2, 3, 4, 16]), near_k, near_v, **c.kw_args)
    for t, s in enumerate(slots.tolist()[:5]):
        assert torch.equal(kc[s // 16, :, :, s % 16], near_k[0, :, :, t]) and torch.equal(vc[s // 16, :, s % 16], near_v[0, :, t])
        assert near_k[0, :, :, t].any() and near_v[0, :, t].any()
    assert torch.count_nonzero(vc.view(NB, -1).any(1)) == 4 and torch.count_nonzero(kc.view(NB, -1).any(1)) == 4


# ------------------------------------------------------------- block tables --

def test_ids_and_slots_up_to_the_last():
    """2^27 blocks: the last slot is 2^31 - 1."""
    NB = 1 << 27
    free = torch.zeros(NB, dtype=torch.int32, device="cuda")
    free[:3] = i32([NB - 3, NB - 2, NB - 1])
    pool = pda.make_block_pool(i32([[-1, -1, -1]]), i32([0]), free, i32([3, 0]))
    positions, slots = i32([0] * 4), i32([0] * 4)
    pda.pda_blocks_resize(pool, i32([18]), positions=positions, slots=slots)
    assert positions.tolist() == [14, 15, 16, 17]
    assert slots.tolist() == [2 ** 31 - 2, 2 ** 31 - 1, 16 * (NB - 2), 16 * (NB - 2) + 1]


@pytest.mark.parametrize("B,width", [(1024, 2500), (1024, 3)])
def test_the_most_sequences_of_one_launch(B, width):
    rng = np.random.RandomState(width)
    pool, model = pda.new_block_pool(B, 30 * B, width), ref.Pool(B, 30 * B, width)
    for step in range(3):
        lens = rng.randint(0, 16 * min(width, 25), B) * (rng.random(B) < 0.7)
        slots = i32(np.zeros(2 * B))
        pda.pda_blocks_resize(pool, i32(lens), slots=slots)
        model.resize(lens)
        table, held, free, counts = (t.cpu().numpy() for t in pool.tensors)
        np.testing.assert_array_equal(table, model.table)
        np.testing.assert_array_equal(held, model.held)
        np.testing.assert_array_equal(free[:counts[0]], model.free)
        np.testing.assert_array_equal(slots.cpu().numpy(), model.slot_map(lens, 2 * np.arange(B + 1), 2 * B)[1])


@pytest.mark.parametrize("B,n", [(1, 9), (40, 500), (40, 70000), (1100, 900)])
def test_contradicting_contents_stay_inside_the_buffers(B, n):
    """Counts, lengths, ids and row starts of any value: nothing outside the pool's buffers is written."""
    rng = np.random.RandomState(B + n)
    NB, width, guard = 50, 7, 64
    wild = lambda size: rng.choice([-2 ** 31, -1, 0, 1, 3, 6, 7, 8, 49, 50, 51, 1000, 2 ** 30, 2 ** 31 - 1], size)
    sizes = dict(table=B * width, held=B, free=NB, counts=2, positions=n, slots=n)
    for trial in range(4):
        arena = i32(np.full(sum(sizes.values()) + guard * (len(sizes) + 1), 12345))
        part, at, spare = {}, guard, torch.ones_like(arena, dtype=torch.bool)
        for name, size in sizes.items():
            part[name] = arena[at:at + size]
            part[name].copy_(i32(wild(size)))
            spare[at:at + size] = False
            at += size + guard
        pool = pda.make_block_pool(part["table"].view(B, width), part["held"], part["free"], part["counts"])
        lens, start = i32(wild(B)), i32(wild(B + 1) if trial % 2 else np.linspace(0, n, B + 1))
        pda.pda_blocks_resize(pool, lens, start, part["positions"], part["slots"])
        pda.pda_slot_map(part["table"].view(B, width), lens, NB, start, part["positions"], part["slots"])
        torch.cuda.synchronize()
        assert (arena[spare] == 12345).all()
        held, counts = part["held"].cpu().numpy(), part["counts"].tolist()
        assert (held >= 0).all() and (held <= width).all() and 0 <= counts[0] <= NB and counts[1] >= 0


def test_two_graphs_with_one_resize_workspace():
    """Of pools of different sizes, replayed in turns, with other work between."""
    rng = np.random.RandomState(4)
    workspace = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    stream, made = torch.cuda.Stream(), []
    for B, width in ((50, 400), (3, 5), (1200, 4)):
        lens = i32(np.zeros(B))
        pool = pda.new_block_pool(B, 9000, width)
        call = pda.bind_blocks_resize(pool, lens, workspace=workspace, stream=stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        made.append((graph, pool, lens, ref.Pool(B, 9000, width)))
    for turn in range(9):
        graph, pool, lens, model = made[turn % 3]
        new = rng.randint(0, 16 * min(40, model.table.shape[1]) + 1, len(model.held))
        lens.copy_(i32(new))
        graph.replay()
        torch.cuda.synchronize()
        model.resize(new)
        np.testing.assert_array_equal(pool.tensors[0].cpu().numpy(), model.table)
        assert pool.tensors[3].tolist() == [len(model.free), model.short]
