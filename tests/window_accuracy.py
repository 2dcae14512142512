"""How far windowed attention may be from the exact one over a whole call (include/pda_window.h), and
inputs to measure it on.

The probabilities enter the product with V as three bf16 parts, each the top 16 bits of what is
left: with 8 significant bits a part, all 24 of an fp32 value, so the split costs nothing.  What is
left is fp32.  With the inputs below a score (in units of log2) has a root mean square of about 1
and is a sum of D = 128 products, each addition rounding a partial sum (1 / sqrt 2 of the whole on
average) by an error that is uniform within 2^-24: ln 2 sqrt(128 / 2 / 3) 2^-24 = 1.9e-7 of a
probability.  The difference to the running maximum, about 4, is rounded by up to 2^-22: uniform,
ln 2 2^-22 / sqrt 3 = 1.0e-7; the rounded maximum is up to 1.7e-7 off from one step to another,
the same for all tokens between: half of that.  exp2 is good to 2^-23, uniform: 0.7e-7.  The sums
over some 600 tokens, 16 at a time, round 38 times in the product and in the row's sum: sqrt(38 / 3)
2^-24 sqrt 2 = 3.0e-7.  Together 3.9e-7 of the norm, since errors that are independent from token to token
change a result by as much of its norm.

  BAR: 1e-6, two and a half times that.
  Two parts, each rounded to nearest, leave 2^-17 sqrt(4 / 21) of p's binade, 2.4e-6 on average over p's leading digits.
  Two parts cut off leave up to 2^-15 of p, always of one sign: 9e-6."""
import numpy as np

import test_gpu_window as windows

BAR = 1e-6  # of the norm

LENS = [1500, 700, 333, 2100]
WINDOW, SINKS = 512, 5


def inputs(Hq, Hkv, D, n, seed):
    """(q, k, v, table, lens) of a step (test_gpu_window.setup) whose scores have a root mean square of about 1."""
    return windows.setup(len(LENS), Hq, Hkv, D, n, LENS, seed, scale_q=0.6)


def rows(q, k, v, table, lens):
    """For every query row of a KV head's first head: (query, keys and values of the tokens it sees), 64 bits."""
    q, k, v = (x.double().numpy() for x in (q, k, v))
    B, n, Hq, _ = q.shape
    G = Hq // k.shape[1]
    for b, L in enumerate(lens):
        for i in range(n):
            p = L - n + i
            t = np.arange(p + 1)
            t = t[(t > p - WINDOW) | (t < SINKS)]
            for g in range(k.shape[1]):
                at = (table[b, t // 16], g, t % 16)
                yield q[b, i, g * G], k[at], v[at]
