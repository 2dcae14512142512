"""Slot maps whose outputs lie over what the call reads, or over each other, are refused before any launch: workgroups
read lengths while others write rows."""
import ctypes

import pytest
import torch

import paper_2405_11143_amd as pda
from paper_2405_11143_amd import pda as P

B, NB, WIDTH, N = 3, 40, 4, 6
TABLE, HELD, FREE, COUNTS, LENS, START, POSITIONS, SLOTS, WORKSPACE = range(1 << 16, 10 << 16, 1 << 16)  # addresses that nothing reads
SIZES = {TABLE: B * WIDTH, HELD: B, FREE: NB, COUNTS: 2, LENS: B, START: B + 1}


def resize(positions, slots, start=START):
    pool = P.pda_block_pool(B, NB, WIDTH, TABLE, HELD, FREE, COUNTS)
    rows = P.pda_token_rows(N, start, positions, slots)
    return pda.load_library().pda_blocks_resize(ctypes.byref(pool), LENS, ctypes.byref(rows), WORKSPACE, 1 << 10, None)


def slot_map(positions, slots, start=START):
    rows = P.pda_token_rows(N, start, positions, slots)
    return pda.load_library().pda_slot_map(B, NB, WIDTH, TABLE, LENS, ctypes.byref(rows), None)


def over(buffer, bytes_):
    """Row buffers of N that share their first, last or only some element with the buffer."""
    return [buffer, buffer + bytes_ - 4, buffer - 4 * (N - 1)]


@pytest.mark.parametrize("buffer", [TABLE, HELD, FREE, COUNTS, LENS, START])
def test_rows_over_a_buffer_of_the_call(buffer):
    for at in over(buffer, 4 * SIZES[buffer]):
        assert resize(at, SLOTS) == resize(POSITIONS, at) == resize(at, None) == P.PDA_ERR_VALUE
        if buffer in (TABLE, LENS, START):
            assert slot_map(at, SLOTS) == slot_map(POSITIONS, at) == slot_map(None, at) == P.PDA_ERR_VALUE


def test_rows_over_the_workspace():
    used = ctypes.c_size_t()
    pool = P.pda_block_pool(B, NB, WIDTH, TABLE, HELD, FREE, COUNTS)
    assert pda.load_library().pda_blocks_workspace_bytes(ctypes.byref(pool), ctypes.byref(used)) == P.PDA_OK
    for at in over(WORKSPACE, used.value // 4 * 4):
        assert resize(at, SLOTS) == resize(POSITIONS, at) == P.PDA_ERR_VALUE


def test_positions_over_slots():
    for at in over(POSITIONS, 4 * N):
        assert resize(POSITIONS, at) == slot_map(POSITIONS, at) == P.PDA_ERR_VALUE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the launch is meant to fail: the addresses are nobody's")
@pytest.mark.parametrize("call", [resize, slot_map])
def test_neighbours_are_not_refused(call):
    """Right behind a buffer, and right in front of it."""
    for buffer in (LENS, START):
        for at in (buffer + 4 * SIZES[buffer], buffer - 4 * N):
            assert call(at, SLOTS) == call(POSITIONS, at) == P.PDA_ERR_HIP
    assert call(POSITIONS, POSITIONS + 4 * N) == call(POSITIONS, POSITIONS - 4 * N, None) == P.PDA_ERR_HIP
