"""Plain 64-bit forms of the head norms, the windowed attention and the block tables, and the
errors that the kernels' arithmetic allows (test infrastructure; no code of the library)."""
import math

import numpy as np
import torch

BLOCK = 16
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


# ---------------------------------------------------------- norms and rotation --

def turned(x, positions, inv_freq, axis, interleaved, sign=1.0, magnitude=1.0):
    """Rows x [T, H, D] (64 bits) with their pairs turned; positions [axes, T], axis [R / 2].
    Also the sum of the magnitudes of each element's pair (what rounding errors scale with)."""
    R = 2 * len(inv_freq)
    y, size = x.clone(), x.abs()
    angle = positions.double()[axis.long()].t() * inv_freq  # [T, R / 2]
    c, s = angle.cos()[:, None] * magnitude, sign * angle.sin()[:, None] * magnitude
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size = size.clone()
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    return y, size


def normed(x, weight, eps, offset=0.0):
    """x / sqrt(mean x^2 + eps) * (weight + offset), 64 bits."""
    u = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return u if weight is None else u * (weight.double() + offset)


# Roundings of a normed and turned element, in units of 2^-24 of its pair's magnitudes: the sum of
# squares of up to 512 elements (16 by one thread, then 5 levels) counts half in the root: 11;
# the mean and the root 3; the products with the root and the weight 3; the angle, rounded to
# 2^-25 turns, 2 pi 2^-25 (7 units at most, with sine and cosine); the turn's products and sum 4.
HEAD_UNITS = 32


def head_tolerance(y, size, dtype):
    return HALF_STEP[dtype] * y.abs() + HEAD_UNITS * 2.0 ** -24 * size * (1 + HALF_STEP[dtype])


def head_grad(x, g, weight, eps, offset, positions, inv_freq, axis, interleaved, magnitude=1.0):
    """(dx, the magnitudes its errors scale with, h u per row): the formulas, 64 bits."""
    if inv_freq is None:
        h, size = g, g.abs()
    else:
        h, size = turned(g, positions, inv_freq, axis, interleaved, -1.0, magnitude)
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if weight is None else weight.double() + offset
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u, f = x * r, h * w
    dx = r * (f - u * (f * u).mean(-1, keepdim=True))
    scale = r * (size * w.abs() + u.abs() * (size * w.abs() * u.abs()).mean(-1, keepdim=True))
    return dx, scale, h * u, size * u.abs()


# ------------------------------------------------------------ windowed attention --

def window_attention(q, k_rows, v_rows, table, lens, scale, window, sinks):
    """(out, error allowed per 2^-24 unit) of q [B, n, Hq, D] over caches as rows
    [blocks, Hkv, 16, D], in 64 bits on the host.  Rows that see nothing are zero."""
    B, n, Hq, D = q.shape
    Hkv = k_rows.shape[1]
    G = Hq // Hkv
    out = np.zeros((B, n, Hq, D))
    tol = np.zeros((B, n, Hq, D))
    for b in range(B):
        L = int(lens[b])
        for i in range(n):
            p = L - n + i
            t = np.array([x for x in range(p + 1) if x > p - window or x < sinks], dtype=np.int64)
            if len(t) == 0:
                continue
            ids = table[b, t // BLOCK]
            for g in range(Hkv):
                K, V = k_rows[ids, g, t % BLOCK], v_rows[ids, g, t % BLOCK]
                Q = q[b, i, g * G:(g + 1) * G]
                s = Q @ K.T * scale
                e = np.exp(s - s.max(1, keepdims=True))
                pr = e / e.sum(1, keepdims=True)
                out[b, i, g * G:(g + 1) * G] = pr @ V
                # a score's rounding: D products and sums, then the scale (natural logarithm)
                off = (D + 8) * abs(scale) * (np.abs(Q) @ np.abs(K).T).max(1)
                # a probability's and a sum's: 64 and one per 16 tokens
                tol[b, i, g * G:(g + 1) * G] = (pr @ np.abs(V)) * (2 * off + 64 + len(t) / 16)[:, None]
    return out, tol


def cache_of(k_rows, v_rows):
    """The library's caches (bf16) of rows [blocks, Hkv, 16, D]."""
    NB, Hkv, _, D = k_rows.shape
    k = k_rows.view(NB, Hkv, BLOCK, D // 8, 8).transpose(2, 3).contiguous()
    return k, v_rows.contiguous()


# ------------------------------------------------------------------ block tables --

class Pool:
    """A block pool on the host, one id at a time."""

    def __init__(self, num_seqs, num_blocks, width):
        self.table = np.full((num_seqs, width), -1, np.int32)
        self.held = np.zeros(num_seqs, np.int32)
        self.free = list(range(num_blocks - 1, -1, -1))
        self.num_blocks, self.short = num_blocks, 0

    def resize(self, lens):
        width = self.table.shape[1]
        need = [min(-(-max(int(x), 0) // BLOCK), width) for x in lens]
        back = []
        for b, m in enumerate(need):
            back += [int(x) for x in self.table[b, m:self.held[b]]]
            self.held[b] = min(self.held[b], m)
        self.free += back[::-1]
        there, wanted = len(self.free), 0
        for b, m in enumerate(need):
            more = m - int(self.held[b])
            wanted += more
            if more and wanted <= there:
                for j in range(self.held[b], m):
                    self.table[b, j] = self.free.pop()
                self.held[b] = m
        self.short = max(0, wanted - there)

    def slot_map(self, lens, row_start, num_rows):
        return slot_map(self.table, self.held, lens, row_start, num_rows, self.num_blocks)


def slot_map(table, held, lens, row_start, num_rows, num_blocks):
    positions, slots = np.full(num_rows, -1, np.int32), np.full(num_rows, -1, np.int32)
    width = table.shape[1]
    for b in range(len(lens)):
        L = min(max(int(lens[b]), 0), BLOCK * width)
        count = int(row_start[b + 1]) - int(row_start[b])
        for i in range(count):
            t = L - count + i
            if t < 0:
                continue
            r, j = int(row_start[b]) + i, t // BLOCK
            positions[r] = t
            if j < held[b] and 0 <= table[b, j] < num_blocks:
                slots[r] = table[b, j] * BLOCK + t % BLOCK
    return positions, slots
