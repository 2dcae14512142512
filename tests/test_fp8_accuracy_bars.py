"""What the accuracy bars of attention over the 8-bit cache tell apart (no GPU): the splits
of the probabilities that the kernels use pass with room, coarser ones fail."""
import numpy as np
import pytest

import fp8_accuracy as acc


def cut(x):
    """The top 16 bits of an fp32 value: 8 significant bits, towards zero."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 1e-300)))
    return np.trunc(x / 2.0 ** (e - 7)) * 2.0 ** (e - 7)


def parts(p, steps):
    total, left = 0.0, p
    for step in steps:
        x = step(left)
        total, left = total + x, left - x
    return total


def off(steps, D, seed):
    """Error of the norm that the split alone makes, and the largest of any probability."""
    st, q, K, V, _ = acc.inputs(8, 2, D, 1, seed)
    err = size = worst = 0.0
    for b, g, rows, k, v, limits in acc.sequences(st, q, K, V):
        s = rows @ k.T * st.scale * np.log2(np.e)
        p = np.float32(np.exp2(s - s.max(-1, keepdims=True))).astype(np.float64)
        split = parts(p, steps)
        worst = max(worst, float((np.abs(split - p) / p).max()))
        want, got = p @ v, split @ v
        scale = p.sum(-1, keepdims=True)
        err, size = err + (((got - want) / scale) ** 2).sum(), size + ((want / scale) ** 2).sum()
    return np.sqrt(err / size), worst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_bars_tell_the_splits_apart(D, seed):
    three, each = off([cut, cut, cut], D, seed)
    assert three <= 0.1 * acc.THREE and each <= acc.THREE_EACH
    two, each = off([acc.bf16, acc.bf16], D, seed)
    assert two <= 0.75 * acc.TWO and each <= acc.TWO_EACH
    assert off([cut, cut], D, seed)[0] > 10 * acc.THREE       # a part less
    assert off([cut, acc.bf16], D, seed)[0] > 1.1 * acc.TWO   # the first half cut off
    assert off([acc.bf16], D, seed)[0] > 100 * acc.TWO


def test_the_scores_of_the_inputs_have_the_size_that_the_bars_assume():
    for D in (64, 128):
        st, q, K, V, _ = acc.inputs(8, 2, D, 1, 1)
        s = np.concatenate([(rows @ k.T * st.scale * np.log2(np.e)).ravel() for _, _, rows, k, _, _ in acc.sequences(st, q, K, V)])
        assert 0.7 <= np.sqrt((s ** 2).mean()) <= 1.2
