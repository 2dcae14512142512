"""The 8-bit KV cache and rotary positions on the GPU against the plain 64-bit
definitions of fp8_reference.

Bars.  Rotation: half a step of the output's type (bf16 2^-8, fp32 2^-24,
relative) plus fp8_reference.ROTATION times the pair's size.  Codes of rows that
are not rotated, scale bytes and read-back rows: equal.  Codes of rotated keys:
half an e4m3 step (2^-4 relative, 2^-10 in the subnormals) plus the rotation's
error.  Attention: per element fp8_reference.attention's bound, and 1e-5 of the
output's 2-norm over a whole call (the roundings of the probabilities' second
halves, at most 2^-16 of a probability each, are independent: 2^-16 / sqrt(3) =
8.8e-6 at most of the norm, about half of that on average)."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2405_11143_amd as pda
import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def up(x, dev, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    return t if dtype is None else t.to(dtype)


def upload(cache, dev):
    k, v, s = (up(x, dev) for x in cache)
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s


def download(cache):
    return [x.view(torch.uint8).cpu().numpy() for x in cache]


def f64(t):
    return t.double().cpu().numpy()


def rounded(x, dtype):
    """fp64 values of x rounded to a torch type (what is handed to the GPU)."""
    return f64(torch.from_numpy(np.asarray(x)).to(dtype))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---------------------------------------------------------------- rotary --

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("D,R,Hq,Hkv", [(128, 128, 4, 2), (64, 64, 3, 1), (128, 32, 5, 1), (64, 48, 2, 0), (80, 16, 3, 3),
                                        (24, 16, 1, 1), (512, 512, 2, 1)], ids=str)
@pytest.mark.parametrize("T", [1, 3, 130])
def test_rotary_rows(dev, dtype, interleaved, D, R, Hq, Hkv, T):
    rng = np.random.RandomState(D + R + T)
    pos = rng.randint(0, 5000, T).astype(np.int32)
    pos[-1] = 2 ** 31 - 1  # far positions lose nothing
    if T > 2:
        pos[1] = -1
        pos[2] = 0
    inv, _ = pda.pda_rotary_inv_freq(R, 10000.0)
    m = 1.25 if D == 24 else 1.0
    x = rng.randn(T, Hq + 2 * Hkv + 1, D) * 3
    rows = up(x, dev, dtype)  # fused rows: q, k and more side by side
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hkv] if Hkv else None
    r = pda.make_rotary(up(inv, dev), interleaved=interleaved, magnitude=m)
    before = rows.clone()
    got_q, got_k = pda.pda_rotary_apply(q, up(pos, dev), r, k=k)
    torch.cuda.synchronize()
    assert torch.equal(rows.view(torch.uint8), before.view(torch.uint8))
    for got, src in ((got_q, q), (got_k, k)):
        if src is None:
            assert got is None
            continue
        xs = f64(src)
        want = ref.rotate(xs, np.maximum(pos, 0), inv, interleaved, magnitude=m)
        want[pos < 0] = 0  # an output made by the binding holds zeros in padding rows
        err = np.abs(f64(got) - want)
        bar = half_step(dtype) * np.abs(want) + ref.ROTATION * ref.partner_size(xs, R, interleaved, m)
        bar[..., R:] = 0  # the rest is copied
        print(f"rotary D={D} R={R} T={T}: worst {np.max(err / np.maximum(bar, 1e-30)):.3f} of the bar", flush=True)
        assert (err <= bar).all()
    # in place, the same rows bit for bit; padding rows and neighbours stay
    pda.pda_rotary_apply(q, up(pos, dev), r, k=k, q_out=q, k_out=k)
    torch.cuda.synchronize()
    live = up(pos >= 0, dev)
    assert torch.equal(rows[:, :Hq][live], got_q[live]) and torch.equal(rows[~live], before[~live])
    assert torch.equal(rows[:, Hq + Hkv:], before[:, Hq + Hkv:])


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
def test_rotary_gradient(dev, interleaved):
    """The backward direction is the adjoint: against the formula's gradient and against differences of the GPU's own
    forward rows."""
    rng = np.random.RandomState(3)
    T, H, D, R, m = 37, 3, 64, 32, 1.1
    pos = rng.randint(0, 9000, T).astype(np.int32)
    inv, _ = pda.pda_rotary_inv_freq(R, 500000.0)
    freq, p = up(inv, dev), up(pos, dev)
    fwd = pda.make_rotary(freq, interleaved=interleaved, magnitude=m)
    bwd = pda.make_rotary(freq, interleaved=interleaved, magnitude=m, backward=True)
    x, g = rng.randn(T, H, D).astype(np.float32), rng.randn(T, H, D).astype(np.float32)
    gx, _ = pda.pda_rotary_apply(up(g, dev), p, bwd)
    want = ref.rotate(g.astype(np.float64), pos, inv, interleaved, backward=True, magnitude=m)
    bar = half_step(torch.float32) * np.abs(want) + ref.ROTATION * ref.partner_size(g, R, interleaved, m)
    assert (np.abs(f64(gx) - want) <= bar).all()
    # d<g, rotate(x)>/dx along a direction: the forward is linear, so the difference quotient has no truncation error
    y, _ = pda.pda_rotary_apply(up(x, dev), p, fwd)
    e = rng.randn(T, H, D).astype(np.float32)
    y2, _ = pda.pda_rotary_apply(up(x + e, dev), p, fwd)
    step = f64(up(x + e, dev)) - x.astype(np.float64)
    left = ((f64(y2) - f64(y)) * g).sum((1, 2))
    right = (step * f64(gx)).sum((1, 2))
    size = (ref.partner_size(np.abs(x) + np.abs(e) + np.abs(x + e), R, interleaved, m) * np.abs(g)).sum((1, 2)) + \
        (np.abs(step) * ref.partner_size(g, R, interleaved, m)).sum((1, 2))
    assert (np.abs(left - right) <= (ref.ROTATION + 2.0 ** -24) * size).all()


def test_rotary_empty_and_many_tokens(dev):
    inv, _ = pda.pda_rotary_inv_freq(16)
    r = pda.make_rotary(up(inv, dev))
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=dev)
    out, _ = pda.pda_rotary_apply(q, torch.zeros(0, dtype=torch.int32, device=dev), r)
    assert out.shape == (0, 2, 64)
    # more tokens than a launch has workgroups
    T = (1 << 20) + 77
    pos = torch.arange(T, dtype=torch.int32, device=dev)
    q = torch.randn(T, 1, 16, device=dev)
    out, _ = pda.pda_rotary_apply(q, pos, r)
    a = pos.double()[:, None] * r.tensor
    want = torch.cat([q[:, 0, :8].double() * a.cos() - q[:, 0, 8:].double() * a.sin(),
                      q[:, 0, 8:].double() * a.cos() + q[:, 0, :8].double() * a.sin()], 1)
    size = q[:, 0, :8].abs() + q[:, 0, 8:].abs()
    assert ((out[:, 0].double() - want).abs() <= (ref.ROTATION + 2.0 ** -23) * torch.cat([size, size], 1)).all()


# ---------------------------------------------------------------- append --

def append_inputs(lens, n, Hq, Hkv, D, seed, dev):
    rng = np.random.RandomState(seed)
    B = len(lens)
    st = W.custom_structure(B, Hq, Hkv, D, [max(x, 0) for x in lens], seed=seed)
    q = rounded(rng.randn(B, n, Hq, D) * 2, torch.bfloat16)
    k = rounded(rng.randn(B, n, Hkv, D) * np.exp2(rng.randint(-3, 4, (B, n, Hkv, 1))), torch.bfloat16)
    v = rounded(rng.randn(B, n, Hkv, D), torch.bfloat16)
    return st, q, k, v


def check_append(st, lens, q, k, v, dev, rot, inv, bad=(), in_place=False):
    """Appends and compares every byte of the cache and every query row."""
    B, n, Hkv, D = k.shape
    cache = ref.empty_cache(st.num_blocks, Hkv, D)
    on_gpu = upload(cache, dev)
    table = st.block_table.copy()
    for b, j, value in bad:
        table[b, j] = value
    bf = torch.bfloat16
    kw = dict(max_context_len=max(st.max_context_len, 1))
    qd = None
    if rot is not None:
        qd = up(q, dev, bf)
        q_out = qd if in_place else torch.full(q.shape, 7.0, dtype=bf, device=dev)
        kw.update(rotary=rot, q=qd, q_out=q_out)
    else:
        kw.update(num_q_heads=q.shape[2])
    got_q = pda.pda_append_kv_fp8(up(k, dev, bf), up(v, dev, bf), up(table, dev), up(np.asarray(lens, np.int32), dev),
                                  *on_gpu, **kw)
    torch.cuda.synchronize()
    got = download(on_gpu)
    R = 0 if rot is None else rot.rotary_dim
    inter = bool(rot is not None and rot.interleaved)
    seen = [np.zeros(c.shape, bool) for c in cache]  # bytes that a new row owns
    for b, L in enumerate(lens):
        L = min(max(L, 0), kw["max_context_len"])
        for i in range(n):
            t = L - n + i
            if rot is not None:
                row = f64(got_q[b, i])
                if t < 0:
                    assert np.array_equal(row, q[b, i] if in_place else np.full_like(row, 7.0))
                else:
                    want = ref.rotate(q[b, i], t, inv, inter, magnitude=rot.magnitude)
                    bar = 2.0 ** -8 * np.abs(want) + ref.ROTATION * ref.partner_size(q[b, i], R, inter, rot.magnitude)
                    assert (np.abs(row - want) <= bar).all(), (b, i)
            if t < 0:
                continue
            page, o = table[b, t // 16], t % 16
            if not 0 <= page < st.num_blocks:
                continue
            for which, x in ((0, k[b, i]), (1, v[b, i])):
                slack = 0.0
                if which == 0 and rot is not None:
                    slack = ref.ROTATION * ref.partner_size(x, R, inter, rot.magnitude)
                    x = ref.rotate(x, t, inv, inter, magnitude=rot.magnitude)
                codes, s = ref.rows(got, page, o, which)
                want_codes, want_s = ref.quantise(x)
                if which == 1 or rot is None:
                    assert np.array_equal(codes, want_codes) and np.array_equal(s, want_s), (b, i, which)
                else:
                    top = np.abs(x).max(-1)
                    edge = 448 * ref.factor(np.minimum(want_s, s))
                    assert ((s == want_s) | (np.abs(top - edge) <= 2.0 ** -18 * top)).all()
                    f = ref.factor(s)[:, None]
                    bar = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * f) + slack * (1 + 2.0 ** -4)
                    assert (np.abs(ref.dequantise(codes, s) - x) <= bar).all(), (b, i)
                d = np.arange(D)
                place = (ref.k_place if which == 0 else ref.v_place)(d, o)
                seen[which][(page, slice(None)) + place] = True
                seen[2][page, :, which, o] = True
    for which in range(3):  # nothing else was written
        assert (got[which][~seen[which]] == ref.POISON).all()
    return got


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 7, 1), (128, 4, 4), (64, 3, 3)], ids=str)
@pytest.mark.parametrize("n,lens", [(1, [1, 16, 17, 0, 333]), (3, [2, 3, 16, 18, 47]), (17, [16, 17, 40, 5, 0]),
                                    (40, [40, 39, 41, 1, 100])], ids=str)
@pytest.mark.parametrize("kind", ["plain", "half", "interleaved", "part"])
def test_append(dev, D, Hq, Hkv, n, lens, kind):
    st, q, k, v = append_inputs(lens, n, Hq, Hkv, D, 100 + n, dev)
    rot, inv = None, None
    if kind != "plain":
        inv, _ = pda.pda_rotary_inv_freq(D if kind != "part" else 48, 10000.0)
        rot = pda.make_rotary(up(inv, dev), interleaved=kind == "interleaved", magnitude=1.5 if kind == "part" else 1.0)
    check_append(st, lens, q, k, v, dev, rot, inv, in_place=kind == "part")


def test_append_special_rows(dev):
    """Zero rows, rows of one value on both sides of a scale's border, subnormals, the largest values, NaN and
    infinities: codes and bytes are those of the definition."""
    D, n = 64, 16
    lens = [20]
    st, q, k, v = append_inputs(lens, n, 2, 2, D, 9, dev)
    x = np.zeros((n, D))
    x[1, 5], x[2, 5], x[3, 5], x[4, 5] = 448, 450, -1.75 * 2.0 ** -40, 1.7578125 * 2.0 ** -40
    x[5, 0], x[6, 0], x[7] = 2.0 ** -133, 2.0 ** -126, 2.0 ** -130 * np.arange(D)
    x[8, 9], x[9] = 3.3895313892515355e38, np.linspace(-3e38, 3e38, D)
    x[10, 3], x[11, 3], x[12, 3] = np.nan, np.inf, -np.inf
    x[13] = -0.0
    x[14] = np.exp2(-np.arange(D) / 3.0)  # from full precision down through the subnormal codes to zero
    x[15] = np.where(np.arange(D) % 37 == 0, 300.0, np.random.RandomState(0).randn(D))
    for h in range(2):
        k[0, :, h] = v[0, :, 1 - h] = rounded(x, torch.bfloat16)
    got = check_append(st, lens, q, k, v, dev, None, None)
    page, o = st.block_table[0, 0], 4 + 10
    assert (ref.rows(got, page, o, 0)[1] == 255).all() and (ref.rows(got, page, o, 0)[0] == 0x7F).all()
    # a non-finite element anywhere makes a rotated key's row NaN too
    inv, _ = pda.pda_rotary_inv_freq(D)
    rot = pda.make_rotary(up(inv, dev))
    cache = upload(ref.empty_cache(st.num_blocks, 2, D), dev)
    pda.pda_append_kv_fp8(up(k, dev, torch.bfloat16), up(v, dev, torch.bfloat16), up(st.block_table, dev),
                          up(np.asarray(lens, np.int32), dev), *cache, rotary=rot, max_context_len=20)
    for i in (10, 11, 12):
        t = 4 + i
        codes, s = ref.rows(download(cache), st.block_table[0, t // 16], t % 16, 0)
        assert (s == 255).all() and (codes == 0x7F).all()


def test_append_bad_blocks_and_clamped_lengths(dev):
    lens = [33, 40, 17, 1000, -5]
    st, q, k, v = append_inputs([33, 40, 17, 48, 0], 20, 4, 2, 64, 11, dev)
    inv, _ = pda.pda_rotary_inv_freq(64)
    rot = pda.make_rotary(up(inv, dev))
    st.block_table[4, 0] = -1
    check_append(st, lens, q, k, v, dev, rot, inv, bad=[(0, 1, -1), (1, 2, st.num_blocks), (2, 0, 2 ** 31 - 1)])


# ------------------------------------------------------------------ read --

def random_cache(st, rng, spread=3):
    """A whole pool of finite codes and scale bytes (some rows zero); slots that no context reaches are NaN."""
    cache = [rng.randint(0, 256, x.shape).astype(np.uint8) for x in ref.empty_cache(st.num_blocks, st.Hkv, st.D)]
    for which in (0, 1):
        cache[which][(cache[which] & 127) == 127] = 0x31
    cache[2] = (119 + rng.randint(-spread, spread + 1, cache[2].shape)).astype(np.uint8)
    live = np.zeros((st.num_blocks, 16), bool)
    for b, L in enumerate(st.context_lens):
        for t in range(L):
            live[st.block_table[b, t // 16], t % 16] = True
    d, o = np.arange(st.D), np.arange(16)[:, None]
    for which, place in ((0, ref.k_place), (1, ref.v_place)):
        at = np.broadcast_arrays(*place(d, o))
        x = cache[which][(slice(None), slice(None)) + tuple(at)]
        x[~np.broadcast_to(live[:, None, :, None], x.shape)] = 0x7F
        cache[which][(slice(None), slice(None)) + tuple(at)] = x
        cache[2][:, :, which][~np.broadcast_to(live[:, None], (st.num_blocks, st.Hkv, 16))] = 255
    return cache


@pytest.mark.parametrize("D,Hkv", [(64, 3), (128, 2), (128, 8)], ids=str)
def test_read(dev, D, Hkv):
    rng = np.random.RandomState(D + Hkv)
    lens = [100, 0, 16, 31, 5, 257]
    st = W.custom_structure(len(lens), Hkv, Hkv, D, lens, seed=5)
    cache = random_cache(st, rng, spread=40)
    cache[2][st.block_table[0, 1], 0, 0, 3] = 0     # a row of zeros
    on_gpu = upload(cache, dev)
    K, V = ref.values(cache, 0), ref.values(cache, 1)
    K[st.block_table[0, 1], 0, 3] = 0
    args = (up(st.block_table, dev), up(st.context_lens, dev))
    for first, count in (([0] * 6, lens), ([37, 0, 3, 30, -4, 0], [29, 5, 13, 7, 20, 1]), ([99, 1, 16, -40, 4, 240], [9] * 6)):
        start = np.concatenate([[2], 2 + np.cumsum(count)]).astype(np.int32)
        rows = int(start[-1]) + 3
        for clip in (rows, rows - 8):
            out = torch.full((2, clip, Hkv, D), 7.0, dtype=torch.bfloat16, device=dev)
            pda.pda_read_kv_fp8(*on_gpu, *args, up(start, dev), out[0], out[1], max_context_len=st.max_context_len,
                                first_token=None if not any(first) else up(np.asarray(first, np.int32), dev))
            want = np.full((2, clip, Hkv, D), 7.0)
            for b, L in enumerate(lens):
                for r in range(start[b], start[b + 1]):
                    t = first[b] + r - start[b]
                    if 0 <= t < L and r < clip:
                        want[0, r], want[1, r] = K[st.block_table[b, t // 16], :, t % 16], V[st.block_table[b, t // 16], :, t % 16]
            assert bool(np.array_equal(f64(out), want))


def test_read_bad_blocks(dev):
    lens = [40, 20]
    st = W.custom_structure(2, 2, 2, 64, lens, seed=6)
    cache = random_cache(st, np.random.RandomState(1))
    table = st.block_table.copy()
    table[0, 1], table[1, 0] = st.num_blocks, -7
    out = torch.full((2, 60, 2, 64), 7.0, dtype=torch.bfloat16, device=dev)
    pda.pda_read_kv_fp8(*upload(cache, dev), up(table, dev), up(st.context_lens, dev), up(np.array([0, 40, 60], np.int32), dev),
                        out[0], out[1], max_context_len=40)
    got = f64(out)
    bad = np.zeros(60, bool)
    bad[16:32] = bad[40:56] = True
    assert np.isnan(got[:, bad]).all() and np.isfinite(got[:, ~bad]).all()


# ---------------------------------------------------------------- decode --

def decode(q, cache, st, dev, n=1, scale=None, **kw):
    return pda.pda_decode_fp8(q, *cache, up(st.block_table, dev), up(st.context_lens, dev),
                              st.scale if scale is None else scale, max_context_len=st.max_context_len, **kw)


def check_decode(got, q, K, V, st, scale, what):
    """Every output row against the definition and its bound."""
    got, q = f64(got), f64(q)
    B, n, Hq, D = q.shape
    G = Hq // st.Hkv
    off = size = 0.0
    worst = 0.0
    for b, L in enumerate(st.context_lens):
        t = np.arange(L)
        page = st.block_table[b, t // 16] if L else np.zeros(0, int)
        for g in range(st.Hkv):
            rows = q[b, :, g * G:(g + 1) * G].reshape(-1, D)
            limits = np.repeat(L - n + 1 + np.arange(n), G)
            want, bound = ref.attention(rows, K[page, g, t % 16], V[page, g, t % 16], limits, scale)
            err = np.abs(got[b, :, g * G:(g + 1) * G].reshape(-1, D) - want)
            assert (err <= bound).all(), (what, b, g, float((err / np.maximum(bound, 1e-300)).max()))
            worst = max(worst, float((err / np.maximum(bound, 1e-300)).max()))
            off, size = off + (err ** 2).sum(), size + (want ** 2).sum()
    rel = np.sqrt(off / size) if size else 0.0
    print(f"{what}: {rel:.2e} of the norm, worst element {worst:.3f} of its bound", flush=True)
    assert rel <= 1e-5, what


def case(lens, Hq, Hkv, D, n, seed, dev, spread=3):
    rng = np.random.RandomState(seed)
    st = W.custom_structure(len(lens), Hq, Hkv, D, lens, seed=seed)
    cache = random_cache(st, rng, spread)
    q = up(rng.randn(len(lens), n, Hq, D) * 1.5, dev, torch.bfloat16)
    K, V = (np.nan_to_num(ref.values(cache, which)) for which in (0, 1))
    return st, cache, q, K, V


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (7, 1), (4, 4), (16, 1), (10, 2)], ids=str)
@pytest.mark.parametrize("n", [1, 2, 5])
@pytest.mark.parametrize("partition_tokens", [0, 16, 80])
def test_decode(dev, D, Hq, Hkv, n, partition_tokens):
    lens = [1, 0, 15, 16, 17, 33, 128, 300]
    st, cache, q, K, V = case(lens, Hq, Hkv, D, n, 40 + n + D, dev)
    on_gpu = upload(cache, dev)
    got = decode(q, on_gpu, st, dev, partition_tokens=partition_tokens)
    check_decode(got, q, K, V, st, st.scale, f"decode D={D} {Hq}/{Hkv} n={n} Tp={partition_tokens}")
    again = decode(q, on_gpu, st, dev, partition_tokens=partition_tokens)
    assert torch.equal(got, again)
    if n == 1:  # the two shapes of a decode step's queries
        flat = decode(q[:, 0], on_gpu, st, dev, partition_tokens=partition_tokens)
        assert torch.equal(flat, got[:, 0])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 17), (8, 1, 8), (7, 1, 19), (4, 4, 33), (12, 2, 22), (16, 1, 9), (8, 2, 70),
                                      (3, 1, 150), (16, 2, 64), (1, 1, 16), (1, 1, 18)], ids=str)
@pytest.mark.parametrize("partition_tokens", [0, 48])
def test_decode_many_new_tokens(dev, D, Hq, Hkv, n, partition_tokens):
    lens = [1, n - 1, n, n + 1, n + 40, 0, 2 * n + 31, 300]
    st, cache, q, K, V = case(lens, Hq, Hkv, D, n, 60 + n + D, dev)
    got = decode(q, upload(cache, dev), st, dev, partition_tokens=partition_tokens)
    check_decode(got, q, K, V, st, st.scale, f"decode D={D} {Hq}/{Hkv} n={n} Tp={partition_tokens}")


@pytest.mark.parametrize("n", [1, 6, 40])
def test_decode_long_contexts(dev, n):
    """Contexts past the 64 block ids a wavefront holds, and more items than run at once."""
    lens = [5000, 4097, 33, 2600] + [300] * 100
    st, cache, q, K, V = case(lens, 8, 4, 64, n, 77, dev)
    got = decode(q, upload(cache, dev), st, dev)
    check_decode(got, q, K, V, st, st.scale, f"long contexts n={n}")


@pytest.mark.parametrize("n", [1, 5, 30])
def test_decode_scales_and_block_placement(dev, n):
    """Scale bytes over a wide range (the largest rows dominate), softmax scales of either sign and zero, and the same
    sequences at other blocks: bit for bit the same."""
    lens = [200, 77, 16, 3]
    for scale, spread in ((0.02, 12), (-0.125, 2), (0.0, 30)):
        st, cache, q, K, V = case(lens, 8, 2, 128, n, 80 + n, dev, spread=spread)
        got = decode(q, upload(cache, dev), st, dev, scale=scale)
        check_decode(got, q, K, V, st, float(np.float32(scale)), f"scale {scale} spread {spread} n={n}")
        perm = np.random.RandomState(1).permutation(st.num_blocks)
        moved = [x[np.argsort(perm)] for x in cache]  # block p moves to perm[p]
        table = np.where(st.block_table >= 0, perm[st.block_table], st.block_table).astype(np.int32)
        other = pda.pda_decode_fp8(q, *upload(moved, dev), up(table, dev), up(st.context_lens, dev), scale,
                                   max_context_len=st.max_context_len)
        assert torch.equal(got, other)


def test_decode_large_values_and_one_token(dev):
    """A context of one token returns its V row exactly, values near the type's largest stay finite, and scores of
    hundreds cancel against their maximum."""
    st, cache, q, K, V = case([1, 40, 64], 4, 2, 128, 1, 91, dev)
    cache[2][:, :, 1] = np.where(cache[2][:, :, 1] == 255, 255, 240)  # V about 2^113 * 448
    K, V = (np.nan_to_num(ref.values(cache, w)) for w in (0, 1))
    got = decode(q, upload(cache, dev), st, dev, scale=3.0)
    check_decode(got, q, K, V, st, 3.0, "large values")
    assert np.array_equal(f64(got)[0, 0], V[st.block_table[0, 0], :, 0].repeat(2, 0))


@pytest.mark.parametrize("n", [1, 6, 40])
def test_decode_bad_blocks(dev, n):
    """A block id outside the pool makes the rows of its sequence that see it NaN, and no others."""
    lens = [100, 120, 90]
    st, cache, q, K, V = case(lens, 8, 2, 64, n, 95, dev)
    st.block_table[1, 2] = st.num_blocks + 5
    for tp in (0, 48):
        got = f64(decode(q, upload(cache, dev), st, dev, partition_tokens=tp))
        assert np.isnan(got[1]).all() and np.isfinite(got[[0, 2]]).all()
    st.block_table[1, 2] = -1
    got = f64(decode(q, upload(cache, dev), st, dev))
    assert np.isnan(got[1]).all() and np.isfinite(got[[0, 2]]).all()


def test_decode_clamps_lengths(dev):
    st, cache, q, K, V = case([60, 20, 33], 4, 2, 64, 2, 96, dev)
    on_gpu = upload(cache, dev)
    want = decode(q, on_gpu, st, dev)
    lens = up(np.array([10 ** 9, 20, 33], np.int32), dev)
    got = pda.pda_decode_fp8(q, *on_gpu, up(st.block_table, dev), lens, st.scale, max_context_len=60)
    assert torch.equal(got, want)
    lens = up(np.array([-3, 20, 33], np.int32), dev)
    got = pda.pda_decode_fp8(q, *on_gpu, up(st.block_table, dev), lens, st.scale, max_context_len=60)
    assert (got[0] == 0).all() and torch.equal(got[1:], want[1:])


def test_decode_matches_the_bf16_cache(dev):
    """The stored values in a bf16 cache give the same attention (fp32 rounding apart)."""
    for n in (1, 5, 40):
        st, cache, q, K, V = case([500, 123, 64, 7], 8, 2, 128, n, 97, dev)
        got = decode(q, upload(cache, dev), st, dev)
        k = W.k_rows_to_cache(up(K, dev, torch.bfloat16))
        other = pda.pda_decode(q, k, up(V, dev, torch.bfloat16), up(st.block_table, dev), up(st.context_lens, dev), st.scale,
                               max_context_len=st.max_context_len)
        assert float((got - other).norm() / other.norm()) <= 2e-5


# ------------------------------------------------------------- together --

def test_a_rollout_over_the_cache(dev):
    """Prompts, then decode steps, the way a rollout runs them: rotate + store, attend, read back at the end."""
    rng = np.random.RandomState(12)
    Hq, Hkv, D, B = 8, 2, 128, 5
    prompts, steps = [30, 1, 64, 17, 45], 6
    final = [p + steps for p in prompts]
    st = W.custom_structure(B, Hq, Hkv, D, final, seed=12)
    table = up(st.block_table, dev)
    cache = upload(ref.empty_cache(st.num_blocks, Hkv, D), dev)
    inv, m = pda.pda_rotary_inv_freq(D, 10000.0, pda.pda.PDA_ROTARY_RAMP, 4.0, 32.0, 1.0, 8.0)
    rot = pda.make_rotary(up(inv, dev), magnitude=m)
    bf = torch.bfloat16
    longest = max(final)
    total = max(prompts)
    qs, ks, vs = (rounded(rng.randn(B, total + steps, H, D), bf) for H in (Hq, Hkv, Hkv))
    outs, at = [], list(prompts)
    chunk = lambda x, lo, hi: up(x[:, lo:hi], dev, bf)
    for step in range(steps + 1):
        n = total if step == 0 else 1
        lo = 0 if step == 0 else total + step - 1
        lens = up(np.asarray(at, np.int32), dev)
        q = chunk(qs, lo, lo + n)
        q_rot = pda.pda_append_kv_fp8(chunk(ks, lo, lo + n), chunk(vs, lo, lo + n), table, lens, *cache, rotary=rot, q=q,
                                      max_context_len=longest)
        outs.append((list(at), n, q_rot, pda.pda_decode_fp8(q_rot, *cache, table, lens, st.scale, max_context_len=longest)))
        at = [x + 1 for x in at]
    torch.cuda.synchronize()
    stored = download(cache)
    K, V = (np.nan_to_num(ref.values(stored, w)) for w in (0, 1))
    for lens, n, q, out in outs:  # later tokens do not change what an earlier step saw
        st.context_lens = np.asarray(lens, np.int32)
        check_decode(out, q, K, V, st, st.scale, f"rollout n={n}")
    # against the unquantised rows: e4m3 rounds each stored value by up to 2^-4
    for b in range(B):
        P = prompts[b]
        pos = np.arange(final[b])
        src = np.concatenate([np.arange(total - P, total), total + np.arange(steps)])
        k_true = ref.rotate(ks[b, src], pos, inv, magnitude=m)
        page = st.block_table[b, pos // 16]
        f = ref.factor(stored[2][page, :, 0, pos % 16])[..., None]
        slack = ref.ROTATION * 1.0625 * ref.partner_size(ks[b, src], D, False, m)
        assert (np.abs(K[page, :, pos % 16] - k_true) <= np.maximum(2.0 ** -4 * np.abs(k_true), 2.0 ** -10 * f) + slack).all()
    # read back
    start = np.concatenate([[0], np.cumsum(final)]).astype(np.int32)
    k_out = torch.empty((int(start[-1]), Hkv, D), dtype=bf, device=dev)
    v_out = torch.empty_like(k_out)
    pda.pda_read_kv_fp8(*cache, table, up(np.asarray(final, np.int32), dev), up(start, dev), k_out, v_out, max_context_len=longest)
    for b in range(B):
        pos = np.arange(final[b])
        page = st.block_table[b, pos // 16]
        assert np.array_equal(f64(k_out[start[b]:start[b + 1]]), K[page, :, pos % 16])
        assert np.array_equal(f64(v_out[start[b]:start[b + 1]]), V[page, :, pos % 16])


def test_captured_step_replays(dev):
    """Rotate + store + attend captured into one graph and replayed over changing lengths, queries and keys, with the
    same work done eagerly (on a cache of its own) between the replays."""
    Hq, Hkv, D, B, first = 8, 2, 64, 6, [1, 30, 64, 200, 15, 90]
    steps = 4
    st = W.custom_structure(B, Hq, Hkv, D, [x + steps for x in first], seed=21)
    table = up(st.block_table, dev)
    start = random_cache(st, np.random.RandomState(2))
    mine, other = upload(start, dev), upload(start, dev)
    inv, _ = pda.pda_rotary_inv_freq(D)
    rot = pda.make_rotary(up(inv, dev))
    bf = torch.bfloat16
    lens = up(np.asarray(first, np.int32), dev)
    q = torch.zeros(B, 1, Hq, D, dtype=bf, device=dev)
    k, v = torch.zeros(2, B, 1, Hkv, D, dtype=bf, device=dev)
    kw = dict(max_context_len=st.max_context_len, partition_tokens=48)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q_rot, out = torch.zeros_like(q), torch.zeros(q.shape, dtype=torch.float32, device=dev)
        store = pda.bind_append_kv_fp8(k, v, table, lens, *mine, rotary=rot, q=q, q_out=q_rot, max_context_len=st.max_context_len)
        attend = pda.bind_decode_fp8(q_rot, *mine, table, lens, st.scale, out, **kw)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            store()
            attend()
    torch.cuda.synchronize()
    for step in range(steps):
        gen = torch.Generator(device=dev)
        gen.manual_seed(step)
        q.copy_(torch.randn(q.shape, generator=gen, device=dev))
        k.copy_(torch.randn(k.shape, generator=gen, device=dev))
        v.copy_(torch.randn(v.shape, generator=gen, device=dev))
        lens.add_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager_q = pda.pda_append_kv_fp8(k, v, table, lens, *other, rotary=rot, q=q, max_context_len=st.max_context_len)
        eager = pda.pda_decode_fp8(eager_q, *other, table, lens, st.scale, **kw)
        torch.cuda.synchronize()
        assert torch.equal(q_rot, eager_q) and torch.equal(out, eager)
        for a, b in zip(mine, other):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_calls_on_another_stream(dev):
    """Calls given a stream run there, in its order."""
    st, cache, q, K, V = case([300, 77, 1], 8, 2, 128, 1, 31, dev)
    want = decode(q, upload(cache, dev), st, dev)
    side = torch.cuda.Stream()
    on_gpu = upload([np.zeros_like(x) for x in cache], dev)
    real = upload(cache, dev)
    table, lens = up(st.block_table, dev), up(st.context_lens, dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for a, b in zip(on_gpu, real):
            a.view(torch.uint8).copy_(b.view(torch.uint8))
    got = pda.pda_decode_fp8(q, *on_gpu, table, lens, st.scale, max_context_len=st.max_context_len, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_empty_batch(dev):
    cache = pda.make_fp8_cache(4, 2, 64, device=dev)
    i32 = dict(dtype=torch.int32, device=dev)
    bf = dict(dtype=torch.bfloat16, device=dev)
    table, lens = torch.zeros(0, 3, **i32), torch.zeros(0, **i32)
    assert pda.pda_decode_fp8(torch.zeros(0, 4, 64, **bf), *cache, table, lens, 0.1, max_context_len=48).shape == (0, 4, 64)
    pda.pda_append_kv_fp8(torch.zeros(0, 1, 2, 64, **bf), torch.zeros(0, 1, 2, 64, **bf), table, lens, *cache, max_context_len=48)
    pda.pda_read_kv_fp8(*cache, table, lens, torch.zeros(1, **i32), torch.zeros(0, 2, 64, **bf), torch.zeros(0, 2, 64, **bf),
                        max_context_len=48)


def test_outputs_made_for_another_stream(dev):
    """Outputs that the binding allocates and clears for a call on a given stream: nothing that the current
    stream still has to do comes after the call's rows."""
    st, cache, q, K, V = case([300, 77, 2], 8, 2, 128, 3, 32, dev)
    rot = pda.make_rotary(up(pda.pda_rotary_inv_freq(128)[0], dev))
    rows, keys = q.reshape(9, 8, 128), up(np.random.RandomState(5).randn(9, 2, 128), dev, torch.bfloat16)
    positions = up(np.array([0, 5, 3, -1, 7, 8, 1000, -2, 4], np.int32), dev)
    new = keys.reshape(3, 3, 2, 128)
    table, lens = up(st.block_table, dev), up(st.context_lens, dev)
    kw = dict(max_context_len=st.max_context_len, rotary=rot, q=q)
    want_rows = pda.pda_rotary_apply(rows, positions, rot, k=keys)
    want_q = pda.pda_append_kv_fp8(new, new, table, lens, *upload(cache, dev), **kw)
    on_gpu = upload(cache, dev)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):  # (a stream, or its handle)
        busy = torch.randn(4096, 4096, device=dev, dtype=torch.bfloat16)
        torch.cuda.synchronize()
        for _ in range(40):
            busy = (busy @ busy).clamp_(-1, 1)
        got_rows = pda.pda_rotary_apply(rows, positions, rot, k=keys, stream=stream)
        got_q = pda.pda_append_kv_fp8(new, new, table, lens, *on_gpu, **kw, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got_rows, want_rows)) and torch.equal(got_q, want_q)


def test_refuses_a_workspace_that_is_not_contiguous(dev):
    st, cache, q, K, V = case([300, 77, 1], 8, 2, 128, 1, 33, dev)
    for ws in (torch.empty(1, dtype=torch.uint8, device=dev).expand(1 << 24),
               torch.empty(1 << 20, dtype=torch.uint8, device=dev)[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            decode(q, upload(cache, dev), st, dev, workspace=ws)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 7, 1), (128, 4, 4)], ids=str)
@pytest.mark.parametrize("n", [1, 4, 13, 60, 200])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("partition_tokens", [0, 48])
def test_decode_rows_of_nan(dev, D, Hq, Hkv, n, which, partition_tokens):
    """A key or value row of NaN inside a context makes the rows that see it NaN, and changes no others (their sums
    do not hold it; the bars of the finite result apply)."""
    lens = [1, n + 3, 250, 297]
    st, cache, q, K, V = case(lens, Hq, Hkv, D, n, 600 + n, dev)
    side = 0 if which == "key" else 1
    hit = [[0], [3, n + 1], [250 - (n + 1) // 2], [296]]  # tokens that only some of the new tokens see, or all
    for b, tokens in enumerate(hit):
        for t in tokens:
            block, slot = st.block_table[b, t // 16], t % 16
            d = np.arange(D)
            place = ref.k_place if side == 0 else ref.v_place
            for g in range(Hkv):
                cache[side][(block, g) + tuple(np.broadcast_arrays(*place(d, slot)))] = 0x7F
                cache[2][block, g, side, slot] = 255
    got = f64(decode(q, upload(cache, dev), st, dev, partition_tokens=partition_tokens))
    limits = np.array(lens)[:, None] - n + 1 + np.arange(n)
    sees = np.array([[any(t < m for t in hit[b]) for m in limits[b]] for b in range(4)])
    assert np.isnan(got[sees]).all() and np.isfinite(got[~sees]).all()
    clean = np.where(sees[:, :, None, None], 0.0, got)
    for b, L in enumerate(lens):
        t = np.arange(L)
        page = st.block_table[b, t // 16]
        for g in range(Hkv):
            rows = f64(q)[b, :, g * (Hq // Hkv):(g + 1) * (Hq // Hkv)].reshape(-1, D)
            want, bound = ref.attention(rows, K[page, g, t % 16], V[page, g, t % 16], np.repeat(limits[b], Hq // Hkv), st.scale)
            keep = np.repeat(~sees[b], Hq // Hkv)
            err = np.abs(clean[b, :, g * (Hq // Hkv):(g + 1) * (Hq // Hkv)].reshape(-1, D) - want)[keep]
            assert (err <= bound[keep]).all()
