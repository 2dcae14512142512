"""Windowed attention where the cache holds infinities and NaN: which rows they reach, at both head
sizes and in every column."""
import numpy as np
import pytest
import torch

import test_gpu_window as windows

pytestmark = pytest.mark.gpu


def sees(t, L, n, window, sinks):
    p = np.arange(L - n, L)
    return (t <= p) & ((t > p - window) | (t < sinks))


# new tokens of 4 heads per KV head: one tile, two, the wide kernel with idle and with full wavefronts
TOKENS = [1, 4, 8, 24, 100]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_value_reaches_the_rows_that_see_it_in_its_column(D, n, bad):
    """Every row of V in a block and every 16-byte piece of it in turn, partly seen and wholly."""
    window, sinks, L = 20, 4, 150
    q, k, v, table, lens = windows.setup(1, 8, 2, D, n, [L], n + D)
    base = windows.run(q, k, v, table, lens, window, sinks).cpu()
    for x, t in enumerate([0, 3] + list(range(max(L - n - 24, 5), L))):
        column = 7 * x % D
        v2 = v.clone()
        v2[table[0, t // 16], 1, t % 16, column] = bad
        got = windows.run(q, k, v2, table, lens, window, sinks).cpu()
        row = sees(t, L, n, window, sinks)
        other = [d for d in range(D) if d != column]
        assert torch.equal(got[0, :, :4], base[0, :, :4]), t  # the other KV head
        assert torch.equal(got[0, ~row, 4:], base[0, ~row, 4:]), t
        assert not torch.isfinite(got[0, row, 4:, column]).any(), t
        assert torch.equal(got[0, row, 4:][..., other], base[0, row, 4:][..., other]), t


@pytest.mark.parametrize("n", TOKENS)
def test_a_bad_key_reaches_the_rows_that_see_it(n):
    window, sinks, L, D = 20, 4, 150, 128
    q, k, v, table, lens = windows.setup(1, 8, 2, D, n, [L], n)
    base = windows.run(q, k, v, table, lens, window, sinks).cpu()
    for x, t in enumerate([0, 3] + list(range(max(L - n - 24, 5), L))):
        k2 = k.clone()
        k2[table[0, t // 16], 1, t % 16, 7 * x % D] = float("nan")
        got = windows.run(q, k2, v, table, lens, window, sinks).cpu()
        row = sees(t, L, n, window, sinks)
        assert torch.equal(got[0, :, :4], base[0, :, :4]) and torch.equal(got[0, ~row, 4:], base[0, ~row, 4:]), t
        assert not torch.isfinite(got[0, row, 4:]).any(), t
