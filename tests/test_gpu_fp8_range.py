"""The ends of the 8-bit cache's range on the GPU: every code under every scale byte, rows
whose largest value rounds up to 2^128, and values of that size in a cache that a caller
filled.  A stored value of 2^128 or more is an infinity: it reads as one, and in the
attention it reaches the rows that see its token and no others."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2405_11143_amd as pda
import workloads as W
from fp8_accuracy import path
from test_gpu_fp8 import case, decode, dev, download, f64, rounded, up, upload  # noqa: F401

pytestmark = pytest.mark.gpu


def stored(x):
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


def as_bf16(x):
    """Values of 4 significant bits (or infinite) as bf16: those below 2^-126 rounded to its subnormals, ties to even."""
    return np.where(np.abs(x) < 2.0 ** -126, np.rint(x * 2.0 ** 133) * 2.0 ** -133, x)


def test_every_code_under_every_scale_byte(dev):  # noqa: F811
    """Read back: exact from 2^-126 up (below, the nearest bf16 subnormal), infinite from 2^128 on; zeros under byte 0,
    NaN under 255 and for NaN codes under the others."""
    D, T = 64, 1024
    cache = ref.empty_cache(T // 16, 1, D)
    for t in range(T):  # token t: scale byte t / 4, codes 64 (t % 4) ..
        for which in (0, 1):
            ref.store(cache, t // 16, t % 16, which, (np.arange(64) + 64 * (t % 4)).astype(np.uint8)[None], np.array([t // 4]))
    table, lens = up(np.arange(T // 16, dtype=np.int32)[None], dev), up(np.array([T], np.int32), dev)
    out = torch.zeros(2, T, 1, D, dtype=torch.bfloat16, device=dev)
    pda.pda_read_kv_fp8(*upload(cache, dev), table, lens, up(np.array([0, T], np.int32), dev), out[0], out[1], max_context_len=T)
    s = np.arange(256)
    want = as_bf16(stored(ref.VALUES * np.where(s == 255, 1.0, 2.0 ** (s - 127.0))[:, None]))
    want[0], want[255] = 0.0, np.nan
    for which in range(2):
        assert np.array_equal(f64(out[which]).reshape(256, 256), want, equal_nan=True)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_near_the_largest_values(dev, D):  # noqa: F811
    """Appended rows of finite values, up to the largest: elements of 1.9375 * 2^127 and more (which round to 2^128, as in
    any format of 4 significant bits) read back infinite, the others within half a step."""
    n, Hkv = 24, 2
    st = W.custom_structure(1, Hkv, Hkv, D, [n], seed=3)
    x = np.random.RandomState(D).uniform(-1, 1, (n, Hkv, D)) * 2.0 ** 127
    top = torch.finfo(torch.bfloat16).max
    x[0, :, 3], x[1, :, 5], x[2, :, 7], x[3, :, 9], x[4] = top, -top, 1.9375 * 2.0 ** 127, 1.9296875 * 2.0 ** 127, top
    x = rounded(np.clip(x, -top, top), torch.bfloat16)
    cache = upload(ref.empty_cache(st.num_blocks, Hkv, D), dev)
    table, lens = up(st.block_table, dev), up(st.context_lens, dev)
    new = up(x[None], dev, torch.bfloat16)
    pda.pda_append_kv_fp8(new, new, table, lens, *cache, max_context_len=n)
    out = torch.zeros(2, n, Hkv, D, dtype=torch.bfloat16, device=dev)
    pda.pda_read_kv_fp8(*cache, table, lens, up(np.array([0, n], np.int32), dev), out[0], out[1], max_context_len=n)
    bytes_ = download(cache)
    t = np.arange(n)
    for which in range(2):
        got = f64(out[which])
        assert np.array_equal(got, stored(ref.values(bytes_, which))[st.block_table[0, t // 16], :, t % 16])
        over = np.abs(x) >= 1.9375 * 2.0 ** 127
        assert np.array_equal(got[over], np.copysign(np.inf, x[over])) and over[2, :, 7].all() and not over[3].any()
        f = ref.factor(bytes_[2][st.block_table[0, t // 16], :, which, t % 16])[..., None]
        assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * f))[~over].all()


@pytest.mark.parametrize("n", [1, 5, 20])
@pytest.mark.parametrize("D", [64, 128])
def test_a_context_of_one_token_at_the_smallest_scales(dev, D, n):  # noqa: F811
    """The attention's rows are then V's, as bf16: subnormals too."""
    for s in (1, 2, 3, 5, 9):
        cache = ref.empty_cache(1, 1, D, fill=0)
        ref.store(cache, 0, 0, 1, np.arange(D).astype(np.uint8)[None] * 2 % 128, np.array([s]))
        q = torch.randn(1, n, 4, D, device=dev).to(torch.bfloat16)
        one = up(np.ones(1, np.int32), dev)
        got = pda.pda_decode_fp8(q, *upload(cache, dev), up(np.zeros((1, 1), np.int32), dev), one, 1.0, max_context_len=1)
        want = as_bf16(ref.VALUES[np.arange(D) * 2 % 128] * 2.0 ** (s - 127))
        assert np.array_equal(f64(got)[0, -1], np.broadcast_to(want, (4, D))) and (f64(got)[0, :-1] == 0).all()


@pytest.mark.parametrize("n", [1, 5, 20, 40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("partition_tokens", [0, 16])
def test_equal_scores_of_any_size_allowed(dev, D, n, partition_tokens):  # noqa: F811
    """Equal scores, up to 2^30 in units of log 2 either way, give the mean of the values: up to 40 of them are summed and
    divided in fp32 (40 + 2 roundings), under probabilities that are off by their parts' error."""
    L = 40
    V = np.random.RandomState(n).randint(0, 120, (L, D)).astype(np.uint8)
    for scale, code, s in ((0.125, 0x38, 127), (0.125, 0x7E, 144), (0.7, 0x7E, 144), (0.7, 0x78, 146), (-0.7, 0x78, 146)):
        size = 4 * abs(scale) * ref.VALUES[code] * 2.0 ** (s - 127) * np.log2(np.e)
        assert size < 2.0 ** 30
        cache = ref.empty_cache(3, 1, D, fill=0)
        for t in range(L):
            k = np.zeros((1, D), np.uint8)
            k[0, 5] = code | 128
            ref.store(cache, t // 16, t % 16, 0, k, np.array([s]))
            ref.store(cache, t // 16, t % 16, 1, V[None, t], np.array([127]))
        q = torch.full((1, n, 4, D), 4.0, dtype=torch.bfloat16, device=dev)
        got = f64(pda.pda_decode_fp8(q, *upload(cache, dev), up(np.arange(3, dtype=np.int32)[None], dev),
                                     up(np.array([L], np.int32), dev), scale, max_context_len=L, partition_tokens=partition_tokens))
        for i in range(n):
            seen = ref.VALUES[V[:L - n + 1 + i]]
            bar = 42 * 2.0 ** -24 + path(n, 4)[1]
            assert (np.abs(got[0, i] - seen.mean(0)) <= bar * np.abs(seen).mean(0)).all(), (scale, s, i)


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
