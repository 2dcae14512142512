"""The 8-bit KV cache and rotary positions on the host (no GPU): the reference's
own pins, the frequencies, and what the entry points refuse before any launch."""
import ctypes
import math

import numpy as np
import pytest

import fp8_reference as ref
import paper_2405_11143_amd as pda
from paper_2405_11143_amd import pda as P


# ---- the reference ----

def test_codes_are_the_nearest_values():
    assert ref.VALUES[0x7E] == 448 and ref.VALUES[0x01] == 2.0 ** -9 and ref.VALUES[0x08] == 2.0 ** -6
    assert np.isnan(ref.VALUES[0x7F]) and np.isnan(ref.VALUES[0xFF])
    finite = np.arange(256)[~np.isnan(ref.VALUES)]
    assert np.array_equal(ref.e4m3_codes(ref.VALUES[finite]), finite)  # (-0 keeps its sign)
    assert list(ref.e4m3_codes(np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10]))) == [0x58, 0x5A, 0x00, 0x02]  # ties


def test_scale_is_the_smallest_power_of_two():
    x = np.zeros((6, 64))
    x[0, 3], x[1, 3], x[2, 3], x[3, 3], x[4, 3] = 448, 448.5, -1.75, 1.76, 2.0 ** -130
    codes, s = ref.quantise(x)
    assert list(s) == [127, 128, 119, 120, 1, 0]
    assert list(codes[:, 3]) == [0x7E, 0x76, 0xFE, 0x76, 0x18, 0]
    y = np.random.RandomState(0).randn(50, 64) * 10.0 ** np.random.RandomState(1).uniform(-30, 30, (50, 1))
    codes, s = ref.quantise(y)
    z = ref.dequantise(codes, s)
    assert (np.abs(z - y) <= np.maximum(np.abs(y) * 2.0 ** -4, 2.0 ** -10 * ref.factor(s)[:, None])).all()


def test_layouts_are_permutations():
    for D in (64, 128):
        d, o = np.arange(D), np.arange(16)[:, None]
        for place, shape in ((ref.k_place, (D // 64, 4, 16, 2, 8)), (ref.v_place, (2, 4, D // 8, 2, 8))):
            flat = np.ravel_multi_index(np.broadcast_arrays(*place(d, o)), shape)
            assert np.array_equal(np.sort(flat.ravel()), np.arange(16 * D))


# ---- the frequencies ----

def test_inv_freq_plain_linear_and_base():
    f, m = pda.pda_rotary_inv_freq(128, 500000.0)
    i = np.arange(64)
    want = 500000.0 ** (-2 * i / 128)
    assert m == 1.0 and np.allclose(f, want, rtol=1e-14, atol=0)
    f, m = pda.pda_rotary_inv_freq(128, 500000.0, P.PDA_ROTARY_LINEAR, 4.0)
    assert m == 1.0 and np.allclose(f, want / 4, rtol=1e-14, atol=0)
    f, m = pda.pda_rotary_inv_freq(128, 500000.0, P.PDA_ROTARY_BASE, 8.0)
    assert f[0] == 1.0 and math.isclose(f[-1], want[-1] / 8, rel_tol=1e-12)  # the lowest divided, the highest kept


def test_inv_freq_bands_and_ramp():
    R, base, factor, orig, low, high = 128, 500000.0, 8.0, 8192.0, 1.0, 4.0
    f, m = pda.pda_rotary_inv_freq(R, base, P.PDA_ROTARY_BANDS, factor, orig, low, high)
    assert m == 1.0
    for i in range(R // 2):
        g = base ** (-2 * i / R)
        wave = 2 * math.pi / g
        if wave < orig / high:
            want = g
        elif wave > orig / low:
            want = g / factor
        else:
            mix = (orig / wave - low) / (high - low)
            want = (1 - mix) * g / factor + mix * g
        assert math.isclose(f[i], want, rel_tol=1e-12), i
    R, base, factor, orig, low, high = 64, 10000.0, 16.0, 4096.0, 1.0, 32.0
    f, m = pda.pda_rotary_inv_freq(R, base, P.PDA_ROTARY_RAMP, factor, orig, low, high)
    assert m == pytest.approx(1 + 0.1 * math.log(16), rel=1e-6)
    turns = orig * base ** (-2 * np.arange(R // 2) / R) / (2 * math.pi)
    plain = base ** (-2 * np.arange(R // 2) / R)
    ratio = f / plain
    assert np.allclose(ratio[turns > high * base ** (2 / R)], 1, rtol=1e-12)
    assert np.allclose(ratio[turns < low / base ** (2 / R)], 1 / factor, rtol=1e-12)
    assert (np.diff(ratio) <= 1e-12).all() and ((ratio > 1 / factor + 0.01) & (ratio < 0.99)).sum() > 3


def test_inv_freq_refusals():
    lib = pda.load_library()
    out = np.zeros(64)
    S = P.pda_rotary_scaling

    def call(R=128, base=1e4, s=None, ptr=out.ctypes.data):
        return lib.pda_rotary_inv_freq(R, base, ctypes.byref(s) if s else None, ptr, None)
    assert call() == P.PDA_OK
    assert call(ptr=None) == P.PDA_ERR_NULL
    for R in (0, -2, 3):
        assert call(R=R) == P.PDA_ERR_SHAPE
    for base in (1.0, 0.5, float("nan"), float("inf")):
        assert call(base=base) == P.PDA_ERR_VALUE
    assert call(s=S(5, 2, 0, 0, 0)) == P.PDA_ERR_UNSUPPORTED
    assert call(s=S(-1, 2, 0, 0, 0)) == P.PDA_ERR_UNSUPPORTED
    for factor in (0.5, 0.0, float("nan"), float("inf")):
        assert call(s=S(1, factor, 0, 0, 0)) == P.PDA_ERR_VALUE
    for kind in (3, 4):
        assert call(s=S(kind, 2, 0, 1, 4)) == P.PDA_ERR_VALUE
        assert call(s=S(kind, 2, 8192, 4, 4)) == P.PDA_ERR_VALUE
        assert call(s=S(kind, 2, 8192, 0, 4)) == P.PDA_ERR_VALUE
    assert call(R=2, s=S(2, 2, 0, 0, 0)) == P.PDA_ERR_SHAPE


# ---- refusals (every call here fails host validation or is empty: nothing is launched) ----

def prob(**kw):
    base = dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=64, num_blocks=128, max_blocks_per_seq=17,
                max_context_len=257)
    base.update(kw)
    return pda.make_problem(**base)


BAD_PROBLEMS = [(dict(num_seqs=-1), P.PDA_ERR_SHAPE), (dict(head_dim=96), P.PDA_ERR_UNSUPPORTED),
                (dict(head_dim=256), P.PDA_ERR_UNSUPPORTED), (dict(block_size=32), P.PDA_ERR_UNSUPPORTED),
                (dict(num_q_heads=34), P.PDA_ERR_UNSUPPORTED), (dict(num_q_heads=7), P.PDA_ERR_SHAPE),
                (dict(max_context_len=17 * 16 + 1), P.PDA_ERR_SHAPE), (dict(num_query_tokens=-1), P.PDA_ERR_SHAPE)]


def rot(**kw):
    base = dict(rotary_dim=64, interleaved=0, backward=0, magnitude=1.0, inv_freq=0x1000)
    base.update(kw)
    return P.pda_rotary(*base.values())


BAD_ROTARY = [(dict(inv_freq=None), P.PDA_ERR_NULL), (dict(rotary_dim=0), P.PDA_ERR_SHAPE),
              (dict(rotary_dim=80), P.PDA_ERR_SHAPE), (dict(rotary_dim=24), P.PDA_ERR_UNSUPPORTED),
              (dict(interleaved=2), P.PDA_ERR_VALUE), (dict(backward=-1), P.PDA_ERR_VALUE),
              (dict(magnitude=float("nan")), P.PDA_ERR_VALUE), (dict(inv_freq=0x1004), P.PDA_ERR_ALIGNMENT)]


def test_rotary_apply_refusals():
    f = pda.load_library().pda_rotary_apply

    def call(r=None, **kw):
        a = dict(T=5, Hq=8, Hkv=2, D=64, dtype=0, pos=0x1000, q=0x1000, qs=512, qo=0x2000, qos=512, k=0x3000, ks=128,
                 ko=0x4000, kos=128)
        a.update(kw)
        r = rot() if r is None else r
        return f(ctypes.byref(r) if r else None, *a.values(), None)
    assert call(r=False) == P.PDA_ERR_NULL
    for kw, status in BAD_ROTARY:
        assert call(rot(**kw)) == status, kw
    for kw in (dict(T=-1), dict(Hq=0), dict(Hkv=-1), dict(D=0), dict(qs=511), dict(qos=504), dict(ks=120), dict(kos=0),
               dict(qo=0x1000, qos=520), dict(ko=0x3000, kos=136), dict(Hq=1 << 30, qs=1 << 40, qos=1 << 40)):
        assert call(**kw) == P.PDA_ERR_SHAPE, kw
    assert call(rot(rotary_dim=16), D=20, Hq=1, Hkv=0) == P.PDA_ERR_UNSUPPORTED
    assert call(rot(rotary_dim=16), D=520, Hq=1, Hkv=0, qs=520, qos=520) == P.PDA_ERR_UNSUPPORTED
    assert call(dtype=2) == P.PDA_ERR_UNSUPPORTED
    for name in ("pos", "q", "qo", "k", "ko"):
        assert call(**{name: None}) == P.PDA_ERR_NULL, name
    for kw in (dict(q=0x1008), dict(qo=0x2002), dict(k=0x3004), dict(ko=0x4008), dict(qs=516), dict(kos=132),
               dict(dtype=1, qs=514)):
        assert call(**kw) == P.PDA_ERR_ALIGNMENT, kw
    assert call(T=0, pos=None, q=None, qo=None, k=None, ko=None) == P.PDA_OK


def test_append_refusals():
    f = pda.load_library().pda_append_kv_fp8

    def call(p=None, r=None, **kw):
        a = dict(q=0x1000, qo=0x2000, k_new=0x3000, v_new=0x4000, bt=0x5000, lens=0x6000, k=0x7000, v=0x8000, s=0x9000)
        a.update(kw)
        return f(ctypes.byref(p or prob()), ctypes.byref(r) if r else None, *a.values(), None)
    for kw, status in BAD_PROBLEMS:
        assert call(prob(**kw), rot()) == status, kw
    assert f(None, *[None] * 10, None) == P.PDA_ERR_NULL
    for kw, status in BAD_ROTARY:
        assert call(r=rot(**kw)) == status, kw
    assert call(r=rot(backward=1)) == P.PDA_ERR_VALUE
    assert call() == P.PDA_ERR_NULL                       # q without a rotation
    assert call(r=rot(), q=None) == P.PDA_ERR_NULL        # one of q and q_out
    assert call(r=rot(), qo=None) == P.PDA_ERR_NULL
    for name in ("k_new", "v_new", "bt", "lens", "k", "v", "s"):
        assert call(r=rot(), **{name: None}) == P.PDA_ERR_NULL, name
    for name in ("q", "qo", "k_new", "v_new", "k", "v", "s"):
        assert call(r=rot(), **{name: 0x1008}) == P.PDA_ERR_ALIGNMENT, name
    assert f(ctypes.byref(prob(num_seqs=0)), *[None] * 10, None) == P.PDA_OK


def test_decode_and_plan_refusals():
    lib = pda.load_library()
    big = 1 << 30

    def call(p=None, scale=0.125, ws=0x9000, ws_bytes=big, **kw):
        a = dict(q=0x1000, k=0x2000, v=0x3000, s=0x4000, bt=0x5000, lens=0x6000)
        out = kw.pop("out", 0x7000)
        a.update(kw)
        return lib.pda_decode_fp8(ctypes.byref(p or prob()), *a.values(), ctypes.c_float(scale), out, ws, ws_bytes, None)
    for kw, status in BAD_PROBLEMS:
        assert call(prob(**kw)) == status, kw
        with pytest.raises(pda.PdaError) as e:
            pda.pda_plan_fp8(prob(**kw))
        assert e.value.status == status
    assert lib.pda_plan_fp8(ctypes.byref(prob()), None) == P.PDA_ERR_NULL
    for name in ("q", "k", "v", "s", "bt", "lens", "out"):
        assert call(**{name: None}) == P.PDA_ERR_NULL, name
    for name in ("q", "k", "v", "s", "out", "ws"):
        assert call(**{name: 0x1008}) == P.PDA_ERR_ALIGNMENT, name
    for scale in (float("nan"), float("inf")):
        assert call(scale=scale) == P.PDA_ERR_VALUE
    need = pda.pda_plan_fp8(prob())["workspace_bytes"]
    assert need > 0
    assert call(ws=None, ws_bytes=0) == P.PDA_ERR_WORKSPACE
    assert call(ws_bytes=need - 1) == P.PDA_ERR_WORKSPACE
    assert lib.pda_decode_fp8(ctypes.byref(prob(num_seqs=0)), *[None] * 6, ctypes.c_float(1), None, None, 0,
                              None) == P.PDA_OK
    # more work items than a launch holds
    with pytest.raises(pda.PdaError) as e:
        pda.pda_plan_fp8(prob(num_seqs=1 << 20, max_blocks_per_seq=1 << 16, max_context_len=1 << 20, partition_tokens=16))
    assert e.value.status == P.PDA_ERR_SHAPE


def test_plan_holds_its_workspace():
    """The workspace: an fp32 state of D + 2 values per output row and partition where contexts are split, then the
    work order."""
    rng = np.random.RandomState(5)
    for _ in range(300):
        D, hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8]))
        G, n, B = int(rng.randint(1, 17)), int(np.exp(rng.uniform(0, 6))), int(rng.randint(0, 300))
        longest = int(np.exp(rng.uniform(0, 9.5)))
        tp = int(rng.choice([0, 0, 16, 48, 256, 1024]))
        try:
            d = pda.pda_plan_fp8(prob(num_seqs=B, num_q_heads=G * hkv, num_kv_heads=hkv, head_dim=D,
                                      max_blocks_per_seq=-(-longest // 16), max_context_len=longest, partition_tokens=tp,
                                      num_query_tokens=n))
        except pda.PdaError as e:
            assert e.status == P.PDA_ERR_SHAPE
            continue
        assert d["partition_tokens"] % 16 == 0 and d["num_partitions"] * d["partition_tokens"] >= longest
        states = B * n * G * hkv * d["num_partitions"] * (D + 2) * 4 if d["num_partitions"] > 1 else 0
        order = d["workspace_bytes"] - states
        assert order >= B * hkv * d["num_partitions"] * 4 and order % 4 == 0


def test_read_refusals():
    f = pda.load_library().pda_read_kv_fp8

    def call(p=None, rows=100, **kw):
        a = dict(k=0x1000, v=0x2000, s=0x3000, bt=0x4000, lens=0x5000, first=0x6000, start=0x7000)
        out = [kw.pop("ko", 0x8000), kw.pop("vo", 0x9000)]
        a.update(kw)
        return f(ctypes.byref(p or prob()), *a.values(), rows, *out, None)
    for kw, status in BAD_PROBLEMS:
        assert call(prob(**kw)) == status, kw
    assert call(rows=-1) == P.PDA_ERR_SHAPE
    for name in ("k", "v", "s", "bt", "lens", "start", "ko", "vo"):
        assert call(**{name: None}) == P.PDA_ERR_NULL, name
    for name in ("k", "v", "s", "ko", "vo"):
        assert call(**{name: 0x1008}) == P.PDA_ERR_ALIGNMENT, name
    assert call(rows=0) == P.PDA_OK
    assert f(ctypes.byref(prob(num_seqs=0)), *[None] * 7, 10, None, None, None) == P.PDA_OK


def test_binding_refusals_without_a_gpu():
    import torch

    k, v, s = pda.make_fp8_cache(4, 2, 64, device="cpu")
    assert k.shape == (4, 2, 1, 4, 16, 2, 8) and v.shape == (4, 2, 2, 4, 8, 2, 8) and s.shape == (4, 2, 2, 16)
    with pytest.raises(ValueError, match="device tensor"):
        pda.make_rotary(torch.zeros(32, dtype=torch.float64))
    with pytest.raises(TypeError, match="float64"):
        pda.make_rotary(torch.zeros(32))
    with pytest.raises(ValueError, match="device tensor"):
        pda.pda_decode_fp8(torch.zeros(1, 4, 64, dtype=torch.bfloat16), k, v, s, torch.zeros(1, 1, dtype=torch.int32),
                           torch.zeros(1, dtype=torch.int32), 0.1, max_context_len=16)
    with pytest.raises(TypeError, match="float8"):
        pda.pda_decode_fp8(torch.zeros(1, 4, 64, dtype=torch.bfloat16), k.view(torch.uint8), v, s,
                           torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0.1,
                           max_context_len=16)
