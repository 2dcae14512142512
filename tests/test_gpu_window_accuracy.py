"""The accuracy that include/pda_window.h states, of the norm over a whole call: decode steps and drafts of one and
of two tiles, steps of the wide kernel, whole and split."""
import numpy as np
import pytest

import test_gpu_window as windows
import window_accuracy as acc
from more_reference import window_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 1), (7, 1, 2), (8, 2, 8), (2, 2, 31),  # 4, 14, 32 and 31 rows of a KV head
                                      (8, 2, 9), (8, 2, 40), (3, 1, 65)], ids=str)  # 36, 160 and 195
@pytest.mark.parametrize("partition_tokens", [0, 96])
def test_accuracy(D, Hq, Hkv, n, partition_tokens):
    q, k, v, table, lens = acc.inputs(Hq, Hkv, D, n, 10 + n)
    want, _ = window_attention(*(x.double().numpy() for x in (q, k, v)), table, lens, D ** -0.5, acc.WINDOW, acc.SINKS)
    got = windows.run(q, k, v, table, lens, acc.WINDOW, acc.SINKS, partition_tokens=partition_tokens).cpu().double().numpy()
    rel = float(np.sqrt(((got - want) ** 2).sum() / (want ** 2).sum()))
    print(f"D={D} {Hq}/{Hkv} n={n} Tp={partition_tokens}: {rel:.2e} of the norm", flush=True)
    assert rel <= acc.BAR


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("partition_tokens", [0, 96])
@pytest.mark.parametrize("size", [8, 24])
def test_larger_scores_add_their_rounding_alone(D, n, partition_tokens, size):
    """Scores `size` times as large, up to about 30 and 90: plain fp32 operations round each once where it is scaled, by up to
    2^-18 at 64 to 128.  The kernels may round a row's maximum by as much beside it, from one step to
    another: no more than twice the error."""
    q, k, v, table, lens = acc.inputs(8, 2, D, n, 30 + n)
    scale = size * D ** -0.5
    in_bits = lambda kind: [x.float().numpy().astype(kind) for x in (q, k, v)]
    want, _ = window_attention(*in_bits(np.float64), table, lens, scale, acc.WINDOW, acc.SINKS)
    plain, _ = window_attention(*in_bits(np.float32), table, lens, scale, acc.WINDOW, acc.SINKS)
    got = windows.run(q, k, v, table, lens, acc.WINDOW, acc.SINKS, scale, partition_tokens=partition_tokens).cpu().double().numpy()
    off = lambda x: float(np.sqrt(((x - want) ** 2).sum() / (want ** 2).sum()))
    print(f"D={D} n={n} Tp={partition_tokens} x{size}: {off(got):.2e} of the norm, plain {off(plain):.2e}", flush=True)
    assert off(got) <= 2 * off(plain) + acc.BAR
