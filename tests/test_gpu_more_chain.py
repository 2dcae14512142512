"""The operators as a rollout engine runs them together, against 64 bits: block tables grown on
the GPU, the slot map's positions and slots, norms and rotation with the keys stored, attention with a
window over what is cached; prompts, then single tokens, a sequence released and another admitted."""
import numpy as np
import pytest
import torch

import paper_2405_11143_amd as pda
from more_reference import normed, turned, window_attention

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (6, 1, 128)])
def test_rollout(Hq, Hkv, D):
    B, NB, width, window, sinks = 4, 60, 12, 40, 4
    gen = torch.Generator().manual_seed(D)
    pool = pda.new_block_pool(B, NB, width)
    kc = torch.full((NB, Hkv, D // 8, 16, 8), float("nan"), dtype=BF, device="cuda")
    vc = torch.full((NB, Hkv, 16, D), float("nan"), dtype=BF, device="cuda")
    inv_freq = torch.from_numpy(10000.0 ** (-2.0 * np.arange(D // 2) / D)).cuda()
    qw, kw = ((1 + 0.2 * torch.randn(D, generator=gen)).to(BF).cuda() for _ in range(2))
    norm, rotary = pda.make_head_norm(qw, kw), pda.make_rotary(inv_freq)
    axis = torch.zeros(D // 2, dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device="cuda")
    history = [[] for _ in range(B)]  # per sequence (k, v) rows in 64 bits, as stored
    lens = [0] * B
    # new tokens per sequence, step by step; -1: released
    for new in ([50, 3, 100, 17], [1, 1, 1, 1], [1, 1, 1, 1], [1, -1, 1, 5], [5, 70, 5, 5], [1, 1, 1, 1]):
        for b, x in enumerate(new):
            if x < 0:
                history[b], lens[b] = [], 0
            else:
                lens[b] += x
        counts = [max(x, 0) for x in new]
        T = sum(counts) + 2  # two rows of padding behind
        positions, slots = i32([9] * T), i32([9] * T)
        pda.pda_blocks_resize(pool, i32(lens), i32(np.concatenate([[0], np.cumsum(counts)])), positions, slots)
        rows = torch.randn((T, Hq + 2 * Hkv, D), generator=gen).to(BF).cuda()
        q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        q_out = pda.pda_norm_rotary_append(q, k, v, positions, slots, kc, vc, norm, rotary)
        # what is stored, read back through the table
        table = pool.tensors[0].cpu().numpy()
        kr, vr = kc.transpose(2, 3).reshape(NB, Hkv, 16, D).double().cpu().numpy(), vc.double().cpu().numpy()
        exact_k = turned(normed(k.double(), kw, 1e-6), positions[None], inv_freq, axis, False)[0].cpu().numpy()
        r = 0
        for b, x in enumerate(counts):
            for t in range(lens[b] - x, lens[b]):
                at = (table[b, t // 16], slice(None), t % 16)
                np.testing.assert_allclose(kr[at], exact_k[r], rtol=2.0 ** -8, atol=2.0 ** -17)
                np.testing.assert_array_equal(vr[at], v[r].double().cpu().numpy())
                history[b].append((kr[at], vr[at]))
                r += 1
        # attention: one call per number of new tokens, over those sequences
        start = np.concatenate([[0], np.cumsum(counts)])
        for x in sorted({c for c in counts if c > 0}):
            which = [b for b, c in enumerate(counts) if c == x]
            qb = torch.stack([q_out[start[b]:start[b] + x] for b in which]).contiguous()
            out = pda.pda_decode_window(qb, kc, vc, pool.tensors[0][which].contiguous(), i32(lens[b] for b in which),
                                        D ** -0.5, window=window, sinks=sinks, max_context_len=16 * width)
            for i, b in enumerate(which):
                n_tok = lens[b]
                blocks = -(-n_tok // 16)
                K, V = np.zeros((blocks, Hkv, 16, D)), np.zeros((blocks, Hkv, 16, D))
                for t, (a, c) in enumerate(history[b]):
                    K[t // 16, :, t % 16], V[t // 16, :, t % 16] = a, c
                want, unit = window_attention(qb[i:i + 1].double().cpu().numpy(), K, V, np.arange(blocks)[None],
                                              [n_tok], D ** -0.5, window, sinks)
                allowed = unit * (2.0 ** -24 + 2.0 ** -15 / 64)
                assert (np.abs(out[i].double().cpu().numpy() - want[0]) <= allowed).all()
    assert int(pool.tensors[3][0]) == NB - sum(-(-x // 16) for x in lens)
