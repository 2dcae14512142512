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
