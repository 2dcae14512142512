"""Attention with a sliding window and sinks against the formula in 64 bits: both kernels, one to
many new tokens, windows of one token to more than the context, sinks inside and outside
the window, contexts shorter than the new tokens, split work, garbage where nothing is seen."""
import numpy as np
import pytest
import torch

import paper_2405_11143_amd as pda
from more_reference import cache_of, window_attention

pytestmark = pytest.mark.gpu

def setup(B, Hq, Hkv, D, n, lens, seed, width=None, spare=3, scale_q=1.5):
    rng = np.random.RandomState(seed)
    lens = np.asarray(lens)
    blocks = [-(-int(x) // 16) for x in lens]
    NB = sum(blocks) + spare
    width = width or max(max(blocks), 1)
    perm, used = rng.permutation(NB), 0
    table = np.full((B, width), -1, np.int32)
    for b, m in enumerate(blocks):
        table[b, :m] = perm[used:used + m]
        used += m
    bf = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
    k = bf(rng.standard_normal((NB, Hkv, 16, D)) + 0.5 * rng.standard_normal((1, Hkv, 1, D)))
    v = bf(rng.standard_normal((NB, Hkv, 16, D)) * np.exp2(rng.standard_normal((NB, Hkv, 16, 1))))
    q = bf(rng.standard_normal((B, n, Hq, D)) * scale_q)
    return q, k, v, table, lens


def seen_mask(lens, n, window, sinks, width):
    """[B, width, 16]: the tokens that some new token sees."""
    t = np.arange(16 * width)
    seen = np.zeros((len(lens), 16 * width), bool)
    for b, L in enumerate(lens):
        for i in range(n):
            p = L - n + i
            if p >= 0:
                seen[b] |= (t <= p) & ((t > p - window) | (t < sinks))
    return seen.reshape(len(lens), width, 16)


def run(q, k, v, table, lens, window, sinks, scale=None, longest=None, **kw):
    kc, vc = cache_of(k, v)
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    longest = 16 * table.shape[1] if longest is None else longest
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    qd = q.cuda() if q.shape[1] > 1 else q[:, 0].contiguous().cuda()
    return pda.pda_decode_window(qd, kc.cuda(), vc.cuda(), dev(table), dev(lens), scale, window=window, sinks=sinks,
                                 max_context_len=longest, **kw).view(q.shape)


def check(q, k, v, table, lens, window, sinks, scale=None, poison=True, **kw):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    f64 = lambda t: t.double().numpy()
    want, unit = window_attention(f64(q), f64(k), f64(v), table, lens, scale, window, sinks)
    if poison:  # whatever nobody sees holds NaN, entries that no seen token has are no block's
        seen = seen_mask(lens, q.shape[1], window, sinks, table.shape[1])
        k, v, table = k.clone(), v.clone(), table.copy()
        keep = np.zeros((k.shape[0], 16), bool)
        for b, j in zip(*np.nonzero(seen.any(2))):
            keep[table[b, j]] |= seen[b, j]
        hidden = torch.from_numpy(~keep)
        k[hidden[:, None].expand(k.shape[:3])] = float("nan")
        v[hidden[:, None].expand(v.shape[:3])] = float("nan")
        table[~seen.any(2)] = 2 ** 30
    got = run(q, k, v, table, lens, window, sinks, scale, **kw).cpu().double().numpy()
    allowed = unit * 2.0 ** -24
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) / np.maximum(allowed, 1e-30))
    assert worst <= 1.0, worst


HEADS = [(8, 2, 64), (4, 1, 128), (6, 6, 64), (14, 2, 128), (16, 1, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 4), (16, 0), (17, 16), (64, 3), (100, 61), (1000, 0), (5, 1000)])
def test_decode(heads, window, sinks):
    lens = [1, 2, 15, 16, 17, 64, 65, 200, 333, 0]
    check(*setup(len(lens), *heads, 1, lens, 7 * window + sinks), window, sinks)


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 2), ((8, 2, 64), 4), ((4, 1, 128), 5), ((8, 2, 128), 8), ((6, 6, 64), 16),
                                     ((6, 6, 64), 31), ((14, 2, 128), 3), ((16, 1, 64), 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (16, 16), (40, 5), (500, 0)])
def test_several_tokens(heads, n, window, sinks):
    lens = [1, 2, n, n + 1, 47, 48, 130, 257, 0]
    check(*setup(len(lens), *heads, n, lens, n), window, sinks)


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 9), ((8, 2, 128), 33), ((4, 4, 64), 70), ((4, 4, 128), 300), ((14, 2, 128), 65),
                                     ((16, 1, 64), 8), ((16, 1, 128), 3), ((3, 1, 128), 129)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (32, 32), (90, 5), (2000, 0)])
def test_wide(heads, n, window, sinks):
    lens = [1, 31, n, n + 40, 515, 0]
    check(*setup(len(lens), *heads, n, lens, n), window, sinks)


@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("partition", [16, 48, 160])
def test_split(n, partition):
    """Few tokens per partition: many partitions, also such that a row sees nothing of."""
    lens = [700, 1, 33, 320]
    check(*setup(4, 8, 2, 128, n, lens, 5), 300, 20, partition_tokens=partition)


@pytest.mark.parametrize("n", [1, 3, 64])
def test_window_past_the_context_is_plain_attention(n):
    q, k, v, table, lens = setup(5, 8, 2, 128, n, [400, 17, 64, 255, 90], 9)
    kc, vc = cache_of(k, v)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    plain = pda.pda_decode(q.cuda(), kc.cuda(), vc.cuda(), dev(np.maximum(table, 0)), dev(lens), 0.1, max_context_len=400)
    got = run(q, k, v, table, lens, 2 ** 31 - 1, 2 ** 31 - 1, 0.1, longest=400)
    # (the plain kernel keeps probabilities to 16 bits)
    assert float((got - plain).abs().max()) <= 2 ** -14 * float(v.abs().max())


@pytest.mark.parametrize("scale", [0.0, -0.2, 30.0, 1e-30])
@pytest.mark.parametrize("n", [1, 4, 24])
def test_scales(n, scale):
    """30: probabilities of one token, the others far below; a masked score stays masked under 0."""
    check(*setup(3, 8, 2, 64, n, [100, 41, 64], 21), 33, 2, scale=scale)


@pytest.mark.parametrize("n", [1, 4, 8, 24, 100])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["k", "v"])
def test_rows_that_do_not_see_a_token_do_not_change(n, bad, which):
    """One element of one token is NaN or infinite: the rows that see it are not finite, all others
    hold what they held: to the bit, except under an infinite score of another row: it moves the reference that
    all rows of its wavefront take their probabilities against, each row's to its own
    maximum so far, which changes their roundings.  Either result is within the tolerance of the exact one, so they
    are within twice that of each other."""
    window, sinks, L = 20, 4, 130
    q, k, v, table, lens = setup(1, 8, 2, 64, n, [L], n)
    base = run(q, k, v, table, lens, window, sinks).cpu()
    unit = window_attention(*(x.double().numpy() for x in (q, k, v)), table, lens, 64 ** -0.5, window, sinks)[1]
    allowed = torch.from_numpy(2 * unit * 2.0 ** -24) if which == "k" and bad == bad else torch.zeros(1, n, 8, 64)
    for t in (2, 5, L - n - 25, L - n - 10, L - n, L - 2, L - 1):
        k2, v2 = k.clone(), v.clone()
        (k2 if which == "k" else v2)[table[0, t // 16], 1, t % 16, 3] = bad
        got = run(q, k2, v2, table, lens, window, sinks).cpu()
        p = np.arange(L - n, L)
        sees = (t <= p) & ((t > p - window) | (t < sinks))
        assert torch.equal(got[0, :, :4], base[0, :, :4])  # the other KV head
        assert ((got[0].double() - base[0].double()).abs() <= allowed[0])[~sees].all(), t
        if which == "v":
            assert not torch.isfinite(got[0, sees, 4:, 3]).any(), t
            other = [d for d in range(64) if d != 3]
            assert torch.equal(got[0, sees, 4:][..., other], base[0, sees, 4:][..., other]), t
        elif bad != bad:
            assert not torch.isfinite(got[0, sees, 4:]).any(), t


def test_bad_block_ids():
    """An id outside the pool where a row looks gives NaN, in rows of that sequence only."""
    for n in (1, 4, 40):
        q, k, v, table, lens = setup(3, 8, 2, 64, n, [100, 100, 100], n)
        table[1, 5] = k.shape[0]
        table[1, 0] = -3  # behind the window: not read
        got = run(q, k, v, table, lens, 33, 0).cpu()
        assert torch.isnan(got[1]).any() and torch.isfinite(got[0]).all() and torch.isfinite(got[2]).all()


def test_one_visible_token_returns_its_value():
    q, k, v, table, lens = setup(4, 8, 2, 128, 1, [1, 16, 17, 200], 1)
    got = run(q, k, v, table, lens, 1, 0).cpu()
    for b, L in enumerate(lens):
        row = v[table[b, (L - 1) // 16], :, (L - 1) % 16].float()
        assert torch.equal(got[b, 0], row.repeat_interleave(4, 0))


@pytest.mark.parametrize("n", [1, 40])
def test_runs_are_reproducible_and_placement_does_not_matter(n):
    q, k, v, table, lens = setup(6, 8, 2, 128, n, [900, 17, 300, 64, 1, 512], 3)
    first = run(q, k, v, table, lens, 200, 7, partition_tokens=64)
    assert torch.equal(first, run(q, k, v, table, lens, 200, 7, partition_tokens=64))
    perm = np.random.RandomState(0).permutation(k.shape[0])
    moved = np.where(table >= 0, perm[np.maximum(table, 0)], -1)
    inv = torch.from_numpy(np.argsort(perm))
    assert torch.equal(first, run(q, k[inv], v[inv], moved, lens, 200, 7, partition_tokens=64))


def test_lengths_are_clamped():
    q, k, v, table, lens = setup(3, 8, 2, 64, 1, [64, 64, 64], 4)
    want = run(q, k, v, table, [64, 0, 64], 20, 2, longest=64)
    assert torch.equal(want, run(q, k, v, table, [2 ** 31 - 1, -5, 65], 20, 2, longest=64))


@pytest.mark.parametrize("n", [1, 40])
def test_captured_on_another_stream(n):
    q, k, v, table, lens = setup(3, 8, 2, 64, n, [300, 41, 64], 8)
    kc, vc = (t.cuda() for t in cache_of(k, v))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    tb, ln, qd = dev(table), dev(lens), q.cuda()
    stream = torch.cuda.Stream()
    call = pda.bind_decode_window(qd, kc, vc, tb, ln, 0.125, window=70, sinks=3, max_context_len=304,
                                  partition_tokens=32, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for new in ([300, 41, 64], [299, 0, 5], [64, 64, 64]):
        ln.copy_(dev(new))
        graph.replay()
        torch.cuda.synchronize()
        want = pda.pda_decode_window(qd, kc, vc, tb, ln, 0.125, window=70, sinks=3, max_context_len=304,
                                     partition_tokens=32)
        # (bit by bit: the last lengths look past a row's blocks, which gives NaN)
        assert torch.equal(call.result.view(torch.int32), want.view(torch.int32))
