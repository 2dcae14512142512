"""Infinities in the 8-bit cache on the GPU: a stored value of 2^128 or more is one, and in
the attention it reaches the rows that see its token and no others."""
import numpy as np
import pytest

import fp8_reference as ref
from test_gpu_fp8 import case, decode, dev, f64, upload  # noqa: F401

pytestmark = pytest.mark.gpu


def stored(x):
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 7, 1), (128, 4, 4)], ids=str)
@pytest.mark.parametrize("n", [1, 4, 13, 60, 200])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("partition_tokens", [0, 48])
def test_attention_over_infinities(dev, D, Hq, Hkv, n, which, partition_tokens):  # noqa: F811
    """A stored infinity changes no row that does not see its token.  Of the rows that see it, a value's element is not
    finite; a key (here under a query element of zero: 0 times infinity) makes the whole row NaN."""
    lens = [1, n + 3, 250, 297]
    st, cache, q, K, V = case(lens, Hq, Hkv, D, n, 700 + n, dev)
    side = 0 if which == "key" else 1
    hit = [[0], [3, n + 1], [250 - (n + 1) // 2], [5, 296]]  # tokens that only some of the new tokens see, or all
    q = q.clone()
    q[..., 0], q[..., 37] = 0, 0
    d = np.arange(D)
    for b, tokens in enumerate(hit):
        for i, t in enumerate(tokens):
            block, slot = st.block_table[b, t // 16], t % 16
            for g in range(Hkv):
                codes = np.zeros(D, np.uint8)
                s = (247, 250, 254)[(b + i + g) % 3]
                codes[(0, 37)[i]] = 0x78 - 8 * (s - 247) | 128 * i  # 2^128 or -2^128
                place = np.broadcast_arrays(*(ref.k_place if side == 0 else ref.v_place)(d, slot))
                cache[side][(block, g) + tuple(place)] = codes
                cache[2][block, g, side, slot] = s
    K, V = (stored(np.nan_to_num(ref.values(cache, w))) for w in (0, 1))
    assert np.isinf((K, V)[side]).any()
    got = f64(decode(q, upload(cache, dev), st, dev, partition_tokens=partition_tokens))
    G, limits = Hq // Hkv, np.array(lens)[:, None] - n + 1 + np.arange(n)
    for b, L in enumerate(lens):
        t = np.arange(L)
        page = st.block_table[b, t // 16]
        rows_limits = np.repeat(limits[b], G)
        blind = rows_limits <= min(hit[b])
        for g in range(Hkv):
            rows = f64(q)[b, :, g * G:(g + 1) * G].reshape(-1, D)
            out = got[b, :, g * G:(g + 1) * G].reshape(-1, D)
            k, v = (np.where(np.isinf(x), 0, x)[page, g, t % 16] for x in (K, V))  # (the blind rows use none of them)
            want, bound = ref.attention(rows[blind], k, v, rows_limits[blind], st.scale)
            assert (np.abs(out[blind] - want) <= bound).all(), (b, g)
            for i, token in enumerate(hit[b]):
                sees = rows_limits > token
                assert np.isnan(out[sees]).all() if side == 0 else not np.isfinite(out[sees][:, (0, 37)[i]]).any()
