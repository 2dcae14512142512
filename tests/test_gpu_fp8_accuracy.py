"""The accuracy that include/pda_fp8.h states for attention over the 8-bit cache, at query
rows on both sides of its line (32 per sequence and KV head): of the norm over a whole
call, and of every element."""
import numpy as np
import pytest

import fp8_accuracy as acc
import fp8_reference as ref
import torch
from test_gpu_fp8 import decode, dev, f64, up, upload  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 1), (7, 1, 1), (16, 1, 2), (8, 2, 5), (8, 1, 4), (2, 2, 32),     # 4 .. 32 rows
                                      (8, 1, 5), (3, 1, 11), (8, 2, 16), (7, 1, 12), (8, 2, 40), (1, 1, 33)],  # 33 .. 160
                         ids=str)
@pytest.mark.parametrize("partition_tokens", [0, 96])
def test_accuracy(dev, D, Hq, Hkv, n, partition_tokens):  # noqa: F811
    st, q, K, V, cache = acc.inputs(Hq, Hkv, D, n, 10 + n)
    norm, each = acc.path(n, Hq // Hkv)
    got = f64(decode(up(q, dev, torch.bfloat16), upload(cache, dev), st, dev, partition_tokens=partition_tokens))
    off = size = 0.0
    for b, g, rows, k, v, limits in acc.sequences(st, q, K, V):
        want, bound = ref.attention(rows, k, v, limits, st.scale)
        spread, _ = ref.attention(rows, k, np.abs(v), limits, st.scale)
        bound = bound - 2 * (2.0 ** -16 - each) * spread  # (its own term for the probabilities' parts)
        G = Hq // Hkv
        err = np.abs(got[b, :, g * G:(g + 1) * G].reshape(-1, D) - want)
        assert (err <= bound).all(), (b, g, float((err / bound).max()))
        off, size = off + (err ** 2).sum(), size + (want ** 2).sum()
    rel = float(np.sqrt(off / size))
    print(f"D={D} {Hq}/{Hkv} n={n} Tp={partition_tokens}: {rel:.2e} of the norm", flush=True)
    assert rel <= norm
