"""Windowed attention where the cache holds infinities and NaN: which rows they reach, at both head
sizes and in every column, and scores of minus infinity, which count nothing."""
import numpy as np
import pytest
import torch

import test_gpu_window as windows
from more_reference import window_attention

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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("partition_tokens", [0, 32])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_scores_of_minus_infinity_count_nothing(D, n, partition_tokens, scale):
    """Keys that score minus infinity in every row leave the rows what they are without those tokens, and
    zero where there is no other; tokens that score plus infinity make the rows that see them non-finite."""
    window, sinks, lens = 40, 4, [150, 61, 17]
    scale *= D ** -0.5
    q, k, v, table, lens = windows.setup(3, 8, 2, D, n, lens, n + D)
    q[..., 5] = 1.0
    k2 = k.clone()
    rng = np.random.RandomState(n)
    gone = [rng.choice(150, 50, replace=False), np.arange(61), np.arange(3, 17)]  # of each sequence; all of the second
    for b, out in enumerate(gone):
        for t in out[out < lens[b]]:
            k2[table[b, t // 16], :, t % 16, 5] = -float("inf") if scale > 0 else float("inf")
    got = windows.run(q, k2, v, table, lens, window, sinks, scale, partition_tokens=partition_tokens).cpu().double().numpy()
    assert np.isfinite(got).all()
    assert (got[1] == 0).all()
    f = lambda x: x.double().numpy()
    K, V, Q = f(k), f(v), f(q)
    for b in (0, 2):
        # the tokens that stay, as a cache of their own for each row: a window over all of it
        for i in range(n):
            p = lens[b] - n + i
            t = np.array([x for x in range(p + 1) if (x > p - window or x < sinks) and x not in gone[b]], dtype=int)
            if len(t) == 0:
                assert (got[b, i] == 0).all()
                continue
            blocks = -(-len(t) // 16)
            kr, vr = np.zeros((blocks, 2, 16, D)), np.zeros((blocks, 2, 16, D))
            x = np.arange(len(t))
            kr[x // 16, :, x % 16], vr[x // 16, :, x % 16] = K[table[b, t // 16], :, t % 16], V[table[b, t // 16], :, t % 16]
            want, unit = window_attention(Q[b:b + 1, i:i + 1], kr, vr, np.arange(blocks)[None], [len(t)], scale, 1000, 0)
            assert (np.abs(got[b, i] - want[0, 0]) <= unit[0, 0] * 2.0 ** -24).all(), (b, i)  # (zeros add without rounding)
    t = 140 - n if n < 100 else 60
    k2 = k.clone()
    k2[table[0, t // 16], :, t % 16, 5] = float("inf") if scale > 0 else -float("inf")
    got = windows.run(q, k2, v, table, lens, window, sinks, scale, partition_tokens=partition_tokens).cpu()
    row = sees(t, lens[0], n, window, sinks)
    assert not torch.isfinite(got[0, row]).any() and torch.isfinite(got[0, ~row]).all() and torch.isfinite(got[1:]).all()
