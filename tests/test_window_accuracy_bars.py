"""What the accuracy bar of windowed attention tells apart (no GPU): three bf16 parts of the
probabilities, with the rest of the arithmetic in fp32, pass with room; two parts fail, however they are
rounded."""
import numpy as np
import pytest

import window_accuracy as acc
from test_fp8_accuracy_bars import cut, parts
from fp8_accuracy import bf16


def off(steps, D, seed):
    """Error of the norm with these parts, scores, exponentials and sums in fp32."""
    err = size = 0.0
    for q, k, v in acc.rows(*acc.inputs(8, 2, D, 4, seed)):
        scale = np.float32(D ** -0.5 * np.log2(np.e))
        s = (k.astype(np.float32) * q.astype(np.float32)).cumsum(1, dtype=np.float32)[:, -1] * scale
        p = np.exp2((s - s.max()).astype(np.float32)).astype(np.float32)
        split = parts(p.astype(np.float64), steps)
        # sums of 16 tokens exactly, then one rounding each
        blocks = np.add.reduceat(split[:, None] * v, np.arange(0, len(p), 16)).astype(np.float32).cumsum(0, dtype=np.float32)[-1]
        total = np.add.reduceat(p.astype(np.float64), np.arange(0, len(p), 16)).astype(np.float32).cumsum(dtype=np.float32)[-1]
        exact = k @ q * (D ** -0.5)
        e = np.exp(exact - exact.max())
        want = e @ v / e.sum()
        err, size = err + ((blocks.astype(np.float64) / float(total) - want) ** 2).sum(), size + (want ** 2).sum()
    return np.sqrt(err / size)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seed", [1, 2])
def test_the_bar_tells_the_splits_apart(D, seed):
    assert off([cut, cut, cut], D, seed) <= 0.75 * acc.BAR
    assert off([bf16, bf16], D, seed) >= 1.75 * acc.BAR
    assert off([cut, bf16], D, seed) >= 1.75 * acc.BAR
    assert off([cut, cut], D, seed) >= 3 * acc.BAR  # a part less


@pytest.mark.parametrize("D", [64, 128])
def test_the_scores_of_the_inputs_have_the_size_that_the_bar_assumes(D):
    s = np.concatenate([k @ q for q, k, _ in acc.rows(*acc.inputs(8, 2, D, 1, 1))]) * D ** -0.5 * np.log2(np.e)
    assert 0.7 <= np.sqrt((s ** 2).mean()) <= 1.2
