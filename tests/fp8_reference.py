"""Plain 64-bit definitions of the 8-bit KV cache and the rotary positions
(include/pda_fp8.h), for the tests: written from the header, sharing nothing
with the kernels."""
import numpy as np

BLOCK = 16
POISON = 0xA9  # a byte that is a finite code and an unlikely scale


def e4m3_values():
    """The value of every code: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinity, NaN at 0x7f."""
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(float) - 10))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


VALUES = e4m3_values()
_POSITIVE = VALUES[:127]  # ascending


def e4m3_codes(y):
    """The codes of values |y| <= 448: nearest, ties to the even code."""
    a = np.abs(y)
    hi = np.searchsorted(_POSITIVE, a).clip(1, 126)
    lo = hi - 1
    d = (a - _POSITIVE[lo]) - (_POSITIVE[hi] - a)
    code = np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantise(x):
    """(codes [..., D], scale bytes [...]) of rows x [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    codes, s = np.zeros(x.shape, np.uint8), np.zeros(x.shape[:-1], np.uint8)
    for i in np.ndindex(*x.shape[:-1]):
        top = np.abs(x[i]).max()
        if not np.isfinite(x[i]).all():
            codes[i], s[i] = 0x7F, 255
            continue
        b = 1
        if top > 0:
            b = max(1, int(np.floor(np.log2(top))) - 10 + 127)
            while top > 448 * 2.0 ** (b - 127):
                b += 1
        s[i] = b if top > 0 else 0
        codes[i] = e4m3_codes(x[i] * 2.0 ** (127 - b))
    return codes, s


def factor(s):
    s = np.asarray(s).astype(np.float64)
    return np.where(s == 255, np.nan, np.where(s == 0, 0.0, 2.0 ** (s - 127)))


def dequantise(codes, s):
    return VALUES[codes] * factor(s)[..., None]


def k_place(d, o):
    """Index of element d of slot o in a K tile's axes [D/64][4][16][2][8]."""
    return d // 64, d // 8 % 4, o, d // 32 % 2, d % 8


def v_place(d, o):
    """... in a V tile's axes [2][4][D/8][2][8]."""
    return o // 2 % 2, o // 4, d // 8, o % 2, d % 8


def empty_cache(num_blocks, hkv, D, fill=POISON):
    return (np.full((num_blocks, hkv, D // 64, 4, BLOCK, 2, 8), fill, np.uint8),
            np.full((num_blocks, hkv, 2, 4, D // 8, 2, 8), fill, np.uint8),
            np.full((num_blocks, hkv, 2, BLOCK), fill, np.uint8))


def store(cache, page, o, which, codes, s):
    """Rows of one token: codes [hkv][D], s [hkv]."""
    d = np.arange(codes.shape[-1])
    place = (k_place if which == 0 else v_place)(d, o)
    cache[which][(page, slice(None)) + place] = codes.T  # (indexed axes apart: they come first)
    cache[2][page, :, which, o] = s


def rows(cache, page, o, which):
    """(codes [hkv][D], s [hkv]) of one token."""
    D = cache[0].shape[2] * 64
    place = (k_place if which == 0 else v_place)(np.arange(D), o)
    return np.ascontiguousarray(cache[which][(page, slice(None)) + place].T), cache[2][page, :, which, o]


def values(cache, which):
    """All rows of the pool as [num_blocks][hkv][16][D] in 64 bits."""
    D = cache[0].shape[2] * 64
    d, o = np.arange(D), np.arange(BLOCK)[:, None]
    place = (k_place if which == 0 else v_place)(d, o)
    place = np.broadcast_arrays(*place)
    codes = cache[which][(slice(None), slice(None)) + tuple(place)]
    return VALUES[codes] * factor(cache[2][:, :, which])[..., None]


def rotate(x, pos, inv_freq, interleaved=False, backward=False, magnitude=1.0):
    """Rows x [..., H, D] at positions pos [...], in 64 bits (angles in longer floats where there are any)."""
    R = 2 * len(inv_freq)
    a = np.asarray(pos)[..., None].astype(np.longdouble) * np.asarray(inv_freq, np.longdouble)
    cos, sin = np.cos(a).astype(np.float64)[..., None, :], np.sin(a).astype(np.float64)[..., None, :]
    if backward:
        sin = -sin
    y = np.array(x, dtype=np.float64)
    first = slice(0, R, 2) if interleaved else slice(0, R // 2)
    second = slice(1, R, 2) if interleaved else slice(R // 2, R)
    p, q = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = magnitude * (p * cos - q * sin), magnitude * (q * cos + p * sin)
    return y


def partner_size(x, R, interleaved, magnitude):
    """m (|x| + |y|) of every element's pair (|x| outside the pairs): what the errors of a rotation scale with."""
    a = np.abs(np.asarray(x, np.float64))
    b = a.copy()
    if interleaved:
        b[..., 0:R:2] = b[..., 1:R:2] = abs(magnitude) * (a[..., 0:R:2] + a[..., 1:R:2])
    else:
        b[..., :R // 2] = b[..., R // 2:R] = abs(magnitude) * (a[..., :R // 2] + a[..., R // 2:R])
    return b


# A rotated element in fp32: two products and a sum (3 roundings), the cosine and sine each within 2 ulp and scaled by
# the magnitude (1 more), the angle's reduction to fp32 turns (half a turn rounded to 24 bits: pi 2^-25 < 2^-23).
ROTATION = (3 + 2 * 3) * 2.0 ** -24 + 2 * 2.0 ** -23


def attention(q, K, V, limits, scale):
    """Softmax attention of rows q [R][D] over K, V [L][D]; row r sees tokens below limits[r].  Returns (out, bound):
    the result and what an fp32 evaluation with the probabilities split in two bf16 halves may be off per element."""
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    R, D = q.shape
    out, bound = np.zeros((R, D)), np.zeros((R, D))
    for r in range(R):
        n = int(min(max(limits[r], 0), len(K)))
        if n == 0:
            continue
        s = scale * (K[:n] @ q[r])
        p = np.exp(s - s.max())
        p /= p.sum()
        out[r] = p @ V[:n]
        # scores: D products summed in fp32, the scaling and the maximum's subtraction; each probability's exponent is
        # off by that much twice (its own and the maximum's), its exp2 by 2^-23, its two halves by 2^-16; the sums of
        # n terms, over partitions too, by n 2^-24 each, the division by 2^-24
        size = abs(scale) * (np.abs(K[:n]) @ np.abs(q[r])).max()
        err = 2 * (D + 4) * 2.0 ** -24 * size + 2.0 ** -16 + (2 * n + 8) * 2.0 ** -24
        bound[r] = 2 * err * (p @ np.abs(V[:n]))
        # fp32 underflow: a probability (over a denominator of at least 1) below 2^-126 may become 0, so may the second
        # half of any, and the result: each at most 2^-126 off, times its value
        bound[r] += 2.0 ** -125 * (1 + np.abs(V[:n]).sum(0))
    return out, bound
