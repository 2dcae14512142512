"""Block tables and slot maps on the GPU against a model that moves one id at a time: growth,
release, shortage, every length from nothing to several spans of entries, odd batches."""
import numpy as np
import pytest
import torch

import paper_2405_11143_amd as pda
from more_reference import Pool, slot_map

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def check_pool(pool, model):
    table, held, free, counts = (t.cpu().numpy() for t in pool.tensors)
    assert counts[0] == len(model.free) and counts[1] == model.short
    np.testing.assert_array_equal(held, model.held)
    np.testing.assert_array_equal(free[:counts[0]], model.free)
    np.testing.assert_array_equal(table, model.table)  # entries past `held` keep what they had
    ids = np.concatenate([free[:counts[0]]] + [table[b, :held[b]] for b in range(len(held))])
    np.testing.assert_array_equal(np.sort(ids), np.arange(len(free)))  # every block once


@pytest.mark.parametrize("B,blocks,width,longest", [(1, 1, 1, 16), (1, 700, 600, 9600), (3, 40, 9, 144), (64, 400, 20, 320),
                                                    (1025, 3000, 12, 192), (2100, 900, 3, 48)])
def test_random_walk(B, blocks, width, longest):
    """Lengths drawn again and again: rows grow, shrink, are released and refused."""
    rng = np.random.RandomState(B + blocks)
    pool, model = pda.new_block_pool(B, blocks, width), Pool(B, blocks, width)
    for step in range(7):
        lens = rng.randint(0, longest + 1, B) * (rng.random(B) < (0.9, 0.3, 1.0)[step % 3])
        if step == 5:
            lens = np.minimum(lens, 17)
        n = rng.randint(0, 40, B)
        start = np.concatenate([[0], np.cumsum(n)])
        rows = int(start[-1]) + 3  # (the last three rows are no sequence's)
        positions, slots = i32(np.full(rows, 77)), i32(np.full(rows, 77))
        pda.pda_blocks_resize(pool, i32(lens), i32(start), positions, slots)
        model.resize(lens)
        check_pool(pool, model)
        want = model.slot_map(lens, start, rows)
        np.testing.assert_array_equal(positions.cpu().numpy(), want[0])
        np.testing.assert_array_equal(slots.cpu().numpy(), want[1])


def test_shortage_grants_in_order():
    pool, model = pda.new_block_pool(5, 10, 8), Pool(5, 10, 8)
    for lens in ([64, 0, 0, 16, 0], [64, 96, 48, 16, 0], [64, 80, 80, 17, 16], [0, 80, 80, 17, 128], [0, 0, 0, 0, 0]):
        pda.pda_blocks_resize(pool, i32(lens))
        model.resize(lens)
        check_pool(pool, model)
    assert model.short == 0 and len(model.free) == 10


def test_grow_and_shrink_is_the_identity():
    """Blocks for drafted tokens, put back when they are rejected: everything as before."""
    rng = np.random.RandomState(3)
    pool = pda.new_block_pool(37, 600, 40)
    lens = rng.randint(1, 200, 37)
    pda.pda_blocks_resize(pool, i32(lens))
    before = [t.clone() for t in pool.tensors]
    count = int(before[3][0])
    pda.pda_blocks_resize(pool, i32(lens + 33))
    grown = pool.tensors[0].clone()
    pda.pda_blocks_resize(pool, i32(lens))
    assert torch.equal(pool.tensors[1], before[1]) and torch.equal(pool.tensors[3], before[3])
    assert torch.equal(pool.tensors[2][:count], before[2][:count])
    pda.pda_blocks_resize(pool, i32(lens + 33))
    assert torch.equal(pool.tensors[0], grown)


@pytest.mark.parametrize("lens", [[-5, 2 ** 31 - 1, 0], [160, 161, -2 ** 31]])
def test_lengths_are_clamped(lens):
    pool, model = pda.new_block_pool(3, 64, 10), Pool(3, 64, 10)
    pos = i32(np.zeros(12))
    pda.pda_blocks_resize(pool, i32(lens), positions=pos)
    model.resize(np.clip(lens, 0, 160))
    check_pool(pool, model)
    np.testing.assert_array_equal(pos.cpu().numpy(), model.slot_map(np.clip(lens, 0, 160), np.arange(4) * 4, 12)[0])


@pytest.mark.parametrize("B,n", [(1, 1), (5, 1), (4, 33), (2, 5000), (3, 30000)])
def test_uniform_rows(B, n):
    """Without row_start every sequence has the same number of rows: positions in front of a short
    context are padding."""
    rng = np.random.RandomState(n)
    lens = rng.randint(0, 2 * n + 3, B)
    pool, model = pda.new_block_pool(B, 1000 * B, 700), Pool(B, 1000 * B, 700)
    positions, slots = i32(np.full(B * n, 9)), i32(np.full(B * n, 9))
    pda.pda_blocks_resize(pool, i32(lens), positions=positions, slots=slots)
    model.resize(lens)
    want = model.slot_map(lens, np.arange(B + 1) * n, B * n)
    np.testing.assert_array_equal(positions.cpu().numpy(), want[0])
    np.testing.assert_array_equal(slots.cpu().numpy(), want[1])


@pytest.mark.parametrize("positions_too", [True, False])
def test_slot_map_of_any_table(positions_too):
    """The map alone: every entry counts, ids outside the pool give no slot."""
    rng = np.random.RandomState(11)
    B, width, blocks = 6, 300, 5000
    table = rng.randint(-2, blocks + 3, (B, width)).astype(np.int32)
    lens = np.array([1, 0, 4800, 16, 17, 4000])
    n = np.array([1, 3, 4800, 20, 0, 1])
    start = np.concatenate([[2], 2 + np.cumsum(n)])  # (the first two rows are no sequence's)
    rows = int(start[-1]) + 5
    positions, slots = i32(np.full(rows, 9)), i32(np.full(rows, 9))
    got = pda.pda_slot_map(i32(table), i32(lens), blocks, i32(start), positions if positions_too else None, slots)
    assert got[1] is slots
    want = slot_map(table, np.full(B, width), lens, start, rows, blocks)
    np.testing.assert_array_equal(slots.cpu().numpy(), want[1])
    np.testing.assert_array_equal(positions.cpu().numpy(), want[0] if positions_too else np.full(rows, 9))


def test_no_sequences():
    pool = pda.new_block_pool(0, 4, 2)
    positions = i32([5, 5])
    pda.pda_blocks_resize(pool, i32([]), row_start=i32([0]), positions=positions)
    assert positions.tolist() == [-1, -1] and pool.tensors[3].tolist() == [4, 0]
    pda.pda_blocks_resize(pool, i32([]))


def test_captured_and_replayed():
    """A resize captured once follows the lengths' current contents."""
    pool, model = pda.new_block_pool(9, 200, 20), Pool(9, 200, 20)
    lens, slots = i32(np.zeros(9)), i32(np.zeros(9))
    call = pda.bind_blocks_resize(pool, lens, slots=slots, stream=(stream := torch.cuda.Stream()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    rng = np.random.RandomState(2)
    for _ in range(4):
        new = rng.randint(0, 200, 9)
        lens.copy_(i32(new))
        graph.replay()
        torch.cuda.synchronize()
        model.resize(new)
        check_pool(pool, model)
        np.testing.assert_array_equal(slots.cpu().numpy(), model.slot_map(new, np.arange(10), 9)[1])


def test_one_workspace_for_several_pools():
    """A workspace of zeros serves one call after the other, on pools of different sizes and both ways of
    running."""
    rng = np.random.RandomState(8)
    pools = [(pda.new_block_pool(B, 4000, width), Pool(B, 4000, width)) for B, width in ((1100, 300), (40, 700), (3, 8))]
    workspace = torch.zeros(32768, dtype=torch.uint8, device="cuda")
    for step in range(3):
        for pool, model in pools:
            lens = rng.randint(0, 100, len(model.held))
            pda.pda_blocks_resize(pool, i32(lens), workspace=workspace)
            model.resize(lens)
            check_pool(pool, model)
