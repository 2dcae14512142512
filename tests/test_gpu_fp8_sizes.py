"""The 8-bit cache and rotary positions at the sizes where their kernels change
course: many tokens, many work items (found by the workgroups themselves or by the
order kernel), contexts past the block ids held at a time, pools past 4 GiB."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2405_11143_amd as pda
import workloads as W
from test_gpu_fp8 import case, check_decode, decode, dev, download, f64, random_cache, rounded, up, upload  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,B,partition_tokens", [
    (16, 16, 64, 50, 0),      # 800 items: 50 pairs, a multiple of 8 KV heads
    (10, 5, 64, 160, 0),      # 800: pairs taken in octets
    (32, 8, 64, 60, 48),      # split contexts: 60 x 4 pairs of 8 heads
    (14, 7, 128, 55, 112),    # 55 x 2 pairs, the last octet of 6
    (24, 24, 64, 43, 32),     # 258 pairs: one too many, the order kernel
    (40, 8, 64, 33, 16),      # 33 x 12 pairs: the order kernel
], ids=str)
@pytest.mark.parametrize("n", [1, 3])
def test_work_orders(dev, Hq, Hkv, D, B, partition_tokens, n):  # noqa: F811
    rng = np.random.RandomState(B)
    lens = rng.randint(0, 190, B)
    lens[:3] = [190, 0, 1]
    st, cache, q, K, V = case(lens.tolist(), Hq, Hkv, D, n, 300 + B, dev)
    plan = pda.pda_plan_fp8(pda.make_problem(B, Hq, Hkv, D, st.num_blocks, st.max_blocks_per_seq, st.max_context_len,
                                             partition_tokens, num_query_tokens=n))
    assert B * Hkv * plan["num_partitions"] > 768
    got = decode(q, upload(cache, dev), st, dev, partition_tokens=partition_tokens)
    check_decode(got, q, K, V, st, st.scale, f"{B} sequences, {plan['num_partitions']} partitions, {Hkv} KV heads, n={n}")


@pytest.mark.parametrize("Hq,Hkv,n,longest,partition_tokens", [
    (6, 1, 7, 4200, 8192),       # 42 rows: two wavefronts, 256 block ids at a time
    (6, 1, 7, 9000, 0),
    (4, 1, 40, 16500, 32768),    # 160 rows: 1024 block ids at a time
    (5, 1, 30, 17000, 0),
    (3, 1, 1, 18000, 32768),     # one wavefront's run past 64 ids
], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_long_contexts(dev, Hq, Hkv, n, longest, partition_tokens, D):  # noqa: F811
    st, cache, q, K, V = case([longest, longest // 2 + 3, n], Hq, Hkv, D, n, 500 + n, dev)
    got = decode(q, upload(cache, dev), st, dev, partition_tokens=partition_tokens)
    check_decode(got, q, K, V, st, st.scale, f"contexts of {longest}, n={n}, D={D}, Tp={partition_tokens}")


@pytest.mark.parametrize("D,R,inter", [(128, 128, False), (128, 64, True), (128, 64, False), (64, 64, False), (256, 128, True)],
                         ids=str)
def test_rotary_many_tokens(dev, D, R, inter):  # noqa: F811
    T, Hq, Hkv = 2500, 5, 2
    inv, _ = pda.pda_rotary_inv_freq(R, 500000.0)
    r = pda.make_rotary(up(inv, dev), interleaved=inter)
    gen = torch.Generator(device=dev)
    gen.manual_seed(D + R)
    rows = torch.randn(T, Hq + 2 * Hkv, D, generator=gen, device=dev).to(torch.bfloat16)
    pos = torch.randint(0, 1 << 20, (T,), generator=gen, device=dev, dtype=torch.int32)
    pos[::97] = -1
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hkv]
    many = pda.pda_rotary_apply(q, pos, r, k=k)
    few = [pda.pda_rotary_apply(q[a:a + 500], pos[a:a + 500], r, k=k[a:a + 500]) for a in range(0, T, 500)]
    for i in range(2):
        assert torch.equal(many[i], torch.cat([f[i] for f in few]))
    sample = np.arange(0, T, 83)
    xs, ps = f64(q[sample]), pos[sample].cpu().numpy()
    want = ref.rotate(xs, np.maximum(ps, 0), inv, inter)
    want[ps < 0] = 0
    bar = 2.0 ** -8 * np.abs(want) + ref.ROTATION * ref.partner_size(xs, R, inter, 1.0)
    assert (np.abs(f64(many[0][sample]) - want) <= bar).all()


@pytest.mark.parametrize("Hq,Hkv,D,R,inter", [(28, 4, 128, 128, False), (8, 2, 128, 128, True), (8, 2, 128, 48, False),
                                              (16, 16, 64, 64, False), (4, 2, 64, 32, True)], ids=str)
def test_append_many_tokens(dev, Hq, Hkv, D, R, inter):  # noqa: F811
    """A batch of many new tokens stores, byte for byte, what its sequences stored one at a time."""
    n, lens = 301, [301, 300, 290, 17, 0, 420, 301, 1, 333]
    st = W.custom_structure(len(lens), Hq, Hkv, D, lens, seed=7)
    inv, _ = pda.pda_rotary_inv_freq(R)
    rot = pda.make_rotary(up(inv, dev), interleaved=inter)
    gen = torch.Generator(device=dev)
    gen.manual_seed(R)
    B = len(lens)
    q = torch.randn(B, n, Hq, D, generator=gen, device=dev).to(torch.bfloat16)
    k, v = torch.randn(2, B, n, Hkv, D, generator=gen, device=dev).to(torch.bfloat16)
    table, ln = up(st.block_table, dev), up(st.context_lens, dev)
    one, other = (upload(ref.empty_cache(st.num_blocks, Hkv, D), dev) for _ in range(2))
    got = pda.pda_append_kv_fp8(k, v, table, ln, *one, rotary=rot, q=q, max_context_len=st.max_context_len)
    for b in range(B):
        s = slice(b, b + 1)
        want = pda.pda_append_kv_fp8(k[s], v[s], table[s], ln[s], *other, rotary=rot, q=q[s], max_context_len=st.max_context_len)
        assert torch.equal(got[s], want)
    for a, b in zip(one, other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # and a token here and there against the definition
    cache = download(one)
    for b, t in ((0, 0), (1, 150), (5, 130), (5, 419), (8, 40)):
        i = t - (lens[b] - n)
        for which, x in ((0, f64(k[b, i])), (1, f64(v[b, i]))):
            slack = 0.0
            if which == 0:
                slack = ref.ROTATION * 1.0625 * ref.partner_size(x, R, inter, 1.0)
                x = ref.rotate(x, t, inv, inter)
            codes, s = ref.rows(cache, st.block_table[b, t // 16], t % 16, which)
            bar = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * ref.factor(s)[:, None]) + slack
            assert (np.abs(ref.dequantise(codes, s) - x) <= bar).all()


def test_pool_past_four_gib(dev):  # noqa: F811
    """Blocks whose offsets pass 32 bits: the same step as in a small pool, bit for bit."""
    Hq, Hkv, D, lens = 16, 8, 128, [70, 33, 16]
    NB = (5 << 30) // (Hkv * 16 * D)  # 5 GiB of K and of V
    st = W.custom_structure(len(lens), Hq, Hkv, D, lens, seed=3)
    far = np.where(st.block_table >= 0, NB - 1 - 7 * st.block_table, -1).astype(np.int32)
    small = upload(random_cache(st, np.random.RandomState(4)), dev)
    big = pda.make_fp8_cache(NB, Hkv, D, device=dev)
    for a, b in zip(big, small):
        a.view(torch.uint8)[NB - 1 - 7 * torch.arange(st.num_blocks, device=dev)] = b.view(torch.uint8)
    inv, _ = pda.pda_rotary_inv_freq(D)
    rot = pda.make_rotary(up(inv, dev))
    ln = up(st.context_lens, dev)
    gen = torch.Generator(device=dev)
    for n in (1, 3, 20):
        gen.manual_seed(n)
        q = torch.randn(3, n, Hq, D, generator=gen, device=dev).to(torch.bfloat16)
        k, v = torch.randn(2, 3, n, Hkv, D, generator=gen, device=dev).to(torch.bfloat16)
        outs = []
        for table, cache in ((up(st.block_table, dev), small), (up(far, dev), big)):
            kw = dict(max_context_len=st.max_context_len)
            qr = pda.pda_append_kv_fp8(k, v, table, ln, *cache, rotary=rot, q=q, **kw)
            out = pda.pda_decode_fp8(qr, *cache, table, ln, st.scale, partition_tokens=32, **kw)
            rows = torch.zeros(2, 119, Hkv, D, dtype=torch.bfloat16, device=dev)
            pda.pda_read_kv_fp8(*cache, table, ln, up(np.array([0, 70, 103, 119], np.int32), dev), rows[0], rows[1], **kw)
            outs.append((out, rows))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        assert bool(torch.isfinite(outs[0][0]).all()) and float(outs[0][1].abs().sum()) > 0


def test_two_steps_at_once(dev):  # noqa: F811
    """Two steps on two streams, each with a workspace of its own, over one cache."""
    st, cache, q, K, V = case([600, 333, 1200, 64], 8, 2, 128, 1, 41, dev)
    on_gpu = upload(cache, dev)
    table, ln = up(st.block_table, dev), up(st.context_lens, dev)
    want = decode(q, on_gpu, st, dev, partition_tokens=64)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls = [pda.bind_decode_fp8(q, *on_gpu, table, ln, st.scale, max_context_len=st.max_context_len, partition_tokens=64,
                                 stream=s) for s in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for call in calls:
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(c.result, want) for c in calls)


def test_seeded_random_steps(dev):  # noqa: F811
    """Random shapes over all variants: append, attend, against the definition."""
    rng = np.random.RandomState(2024)
    for i in range(24):
        D, Hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 3, 8]))
        G = int(rng.randint(1, 17))
        n = int(np.exp(rng.uniform(0, np.log(90))))
        B = int(rng.randint(1, 7))
        lens = [int(np.exp(rng.uniform(0, np.log(500)))) for _ in range(B)]
        tp = int(rng.choice([0, 0, 16, 64, 208]))
        st, cache, q, K, V = case(lens, G * Hkv, Hkv, D, n, 700 + i, dev)
        print(f"random step {i}: D={D} Hkv={Hkv} G={G} n={n} lens={lens} Tp={tp}", flush=True)
        got = decode(q, upload(cache, dev), st, dev, partition_tokens=tp)
        check_decode(got, q, K, V, st, st.scale, f"random step {i}")
