"""How far attention over the 8-bit cache may be from the exact one (include/pda_fp8.h), and
inputs to measure it on.

The probabilities enter the product with V as bf16 parts.  Up to 32 query rows per
sequence and KV head: three parts, each the top 16 bits of what is left, together all 24
bits.  Beyond: two, each rounded to nearest.  bf16 has 8 significant bits, so with p in
[2^e, 2^(e+1)) the first leaves r, uniform within 2^(e-8) on either side, and the second
rounds r to half a step of r's own binade: 2^(e-17) with probability 1/2, half of that
with 1/4, ...: at most 2^-17 of p, and as independent errors a root mean square of 2^(e-17)
sqrt((1/2) (8/7) / 3) = 2^-17 sqrt(4/21) of 2^e, at most that of p.  Relative errors of
that size in the probabilities, independent from token to token, change the result by as
much of its norm.

Everything else is fp32.  With the inputs below a score (in units of log2) has a root mean
square of about 1 and is a sum of D = 128 products, each addition rounding a partial sum
(1/sqrt 2 of the whole on average) by an error that is uniform within 2^-24: ln 2
sqrt(128 / 2 / 3) 2^-24 = 1.9e-7 of a probability.  exp2 is good to 2^-23, uniform: 0.7e-7.
The sums over up to 1024 tokens, 32 at a time, round 32 times: sqrt(32 / 3) 2^-24 =
1.9e-7.  Together 2.8e-7.

  THREE parts: 2.8e-7, bar 6e-7.  (Two parts cut off, not rounded, leave 9e-6: up to 2^-15
  of p, always of one sign.)
  TWO: sqrt(3.33^2 + 0.28^2) e-6 = 3.34e-6, bar 3.6e-6; over p's leading digits it is 2.4e-6
  on average.  (A first part cut off leaves twice the error: 4.7e-6 on average.)"""
import numpy as np

import fp8_reference as ref
import workloads as W

THREE, TWO = 6e-7, 3.6e-6        # of the norm
THREE_EACH, TWO_EACH = 2.0 ** -24, 2.0 ** -17  # of a probability

LENS = [1000, 613, 1024, 257]


def path(n, G):
    """(norm's bar, a probability's own) of n new tokens of G heads per KV head."""
    return (THREE, THREE_EACH) if n * G <= 32 else (TWO, TWO_EACH)


def bf16(x):
    """Values of a bf16 grid: x rounded to 8 significant bits, ties to even."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 1e-300)))
    return np.rint(x / 2.0 ** (e - 7)) * 2.0 ** (e - 7)


def inputs(Hq, Hkv, D, n, seed):
    """(structure, q, K, V, cache): keys with an offset per channel and a few strong channels, values of different sizes
    from token to token; K and V are what the cache holds."""
    rng = np.random.RandomState(seed)
    st = W.custom_structure(len(LENS), Hq, Hkv, D, LENS, seed=seed)
    offset = rng.randn(Hkv, 1, D) * 0.5
    offset[:, :, ::37] *= 6
    k = rng.randn(st.num_blocks, Hkv, 16, D) + offset
    v = rng.randn(st.num_blocks, Hkv, 16, D) * np.exp2(rng.randn(st.num_blocks, Hkv, 16, 1))
    cache = ref.empty_cache(st.num_blocks, Hkv, D)
    d, o = np.arange(D), np.arange(16)[:, None]
    for which, (x, place) in enumerate(((k, ref.k_place), (v, ref.v_place))):
        top = np.abs(x).max(-1)
        s = np.ceil(np.log2(top / 448))
        cache[2][:, :, which] = s + 127
        cache[which][(slice(None), slice(None)) + tuple(np.broadcast_arrays(*place(d, o)))] = ref.e4m3_codes(x * 2.0 ** -s[..., None])
    q = bf16(rng.randn(len(LENS), n, Hq, D) * 0.5)
    return st, q, ref.values(cache, 0), ref.values(cache, 1), cache


def sequences(st, q, K, V):
    """For every sequence and KV head: (b, g, query rows, keys, values, limits)."""
    B, n, Hq, D = q.shape
    G = Hq // st.Hkv
    for b, L in enumerate(st.context_lens):
        t = np.arange(L)
        page = st.block_table[b, t // 16]
        for g in range(st.Hkv):
            yield (b, g, q[b, :, g * G:(g + 1) * G].reshape(-1, D), K[page, g, t % 16], V[page, g, t % 16],
                   np.repeat(L - n + 1 + np.arange(n), G))
