"""Head norms, windowed attention and block tables on the host (no GPU): the reference's own pins, and
what the entry points and the bindings refuse before any launch."""
import ctypes

import numpy as np
import pytest
import torch

import more_reference as ref
import paper_2405_11143_amd as pda
from paper_2405_11143_amd import pda as P

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
SOME = 4096  # an aligned address that nothing reads: every call here is refused, or empty


# ---- the reference ----

def test_normed_and_turned_by_hand():
    x = torch.tensor([[[3.0, 4.0, 0.0, 0.0]]], dtype=torch.float64)
    z = ref.normed(x, torch.tensor([1.0, 2.0, 1.0, 1.0]), 0.0, offset=1.0)
    assert torch.allclose(z, torch.tensor([[[3 / 2.5 * 2, 4 / 2.5 * 3, 0, 0]]], dtype=torch.float64))
    pos = torch.tensor([[1], [3]])
    f = torch.tensor([np.pi / 2, np.pi / 3], dtype=torch.float64)
    axis = torch.tensor([0, 1], dtype=torch.uint8)
    x = torch.tensor([[[1.0, 2.0, 5.0, 7.0]]], dtype=torch.float64)
    y, size = ref.turned(x, pos, f, axis, False)  # pairs (1, 5) by a quarter, (2, 7) by a half
    assert torch.allclose(y, torch.tensor([[[-5.0, -2.0, 1.0, -7.0]]], dtype=torch.float64))
    assert size.tolist() == [[[6.0, 9.0, 6.0, 9.0]]]
    y, _ = ref.turned(x, pos, f, axis, True)  # pairs (1, 2), (5, 7)
    assert torch.allclose(y, torch.tensor([[[-2.0, 1.0, -5.0, -7.0]]], dtype=torch.float64))


def test_gradient_is_the_derivative():
    """The reference's gradient against torch's own, in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((5, 3, 8), generator=gen, dtype=torch.float64, requires_grad=True)
    w = torch.randn(8, generator=gen, dtype=torch.float64, requires_grad=True)
    g = torch.randn((5, 3, 8), generator=gen, dtype=torch.float64)
    pos, f = torch.randint(-5, 9, (2, 5), generator=gen), torch.rand(3, generator=gen, dtype=torch.float64)
    axis = torch.tensor([0, 1, 1], dtype=torch.uint8)
    z = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 0.1) * (w + 1)
    a = (pos[axis.long()].t() * f)[:, None]
    y = torch.cat([z[..., :3] * a.cos() - z[..., 3:6] * a.sin(), z[..., 3:6] * a.cos() + z[..., :3] * a.sin(), z[..., 6:]], -1)
    (y * g).sum().backward()
    dx, _, hu, _ = ref.head_grad(x.detach(), g, w.detach(), 0.1, 1.0, pos, f, axis, False)
    assert torch.allclose(dx, x.grad, atol=1e-12) and torch.allclose(hu.sum((0, 1)), w.grad, atol=1e-12)


def test_window_attention_by_hand():
    """Equal scores: a row is the mean of the values it sees."""
    v = np.arange(16, dtype=np.float64)[None, None, :, None] * np.ones((1, 1, 16, 64))
    q = np.zeros((1, 3, 1, 64))
    out, _ = ref.window_attention(q, np.zeros((1, 1, 16, 64)), v, np.array([[0]]), [12], 1.0, 4, 2)
    assert np.allclose(out[0, :, 0, 0], [np.mean([0, 1, p - 3, p - 2, p - 1, p]) for p in (9, 10, 11)])
    out, _ = ref.window_attention(q, np.zeros((1, 1, 16, 64)), v, np.array([[0]]), [1], 1.0, 4, 2)
    assert np.allclose(out[0, :, 0, 0], [0, 0, 0])  # two rows see nothing, the third token 0


def test_pool_by_hand():
    p = ref.Pool(3, 5, 4)
    p.resize([20, 0, 16])
    assert p.table[0, :2].tolist() == [0, 1] and p.table[2, 0] == 2 and p.free == [4, 3]
    p.resize([20, 48, 16])  # three wanted, two there: none
    assert p.held.tolist() == [2, 0, 1] and p.short == 1
    p.resize([1, 48, 16])  # the block put back is on top
    assert p.table[1, :3].tolist() == [1, 3, 4] and p.short == 0 and p.free == []
    pos, slots = p.slot_map([1, 48, 16], [0, 2, 4, 4], 5)
    assert pos.tolist() == [-1, 0, 46, 47, -1] and slots.tolist() == [-1, 0, 4 * 16 + 14, 4 * 16 + 15, -1]


# ---- refusals of the C entry points ----

def rotary(dim=64, interleaved=0, backward=0, magnitude=1.0, freq=SOME):
    return P.pda_rotary(dim, interleaved, backward, magnitude, freq)


def norm(eps=1e-6, offset=0.0, dtype=0, qw=SOME, kw=SOME):
    return P.pda_head_norm(eps, offset, dtype, qw, kw)


def ref_of(x):
    return ctypes.byref(x) if x is not None else None


def call_norm(n=None, r=None, x=None, T=3, hq=4, hkv=2, D=64, dtype=0, pos=SOME, q=SOME, qs=256, qo=SOME, qos=256,
              k=SOME, ks=128, ko=SOME, kos=128):
    return pda.load_library().pda_norm_rotary(ref_of(n), ref_of(r), ref_of(x), T, hq, hkv, D, dtype, pos, q, qs, qo, qos, k,
                                              ks, ko, kos, None)


SHARED = [  # what every call on head rows refuses
    (dict(D=63), P.PDA_ERR_UNSUPPORTED), (dict(D=0), P.PDA_ERR_SHAPE), (dict(T=-1), P.PDA_ERR_SHAPE),
    (dict(hkv=-1), P.PDA_ERR_SHAPE), (dict(n=norm(eps=-1.0)), P.PDA_ERR_VALUE), (dict(n=norm(eps=float("nan"))), P.PDA_ERR_VALUE),
    (dict(n=norm(offset=float("inf"))), P.PDA_ERR_VALUE), (dict(n=norm(dtype=2)), P.PDA_ERR_UNSUPPORTED),
    (dict(n=norm(qw=SOME + 8)), P.PDA_ERR_ALIGNMENT), (dict(r=rotary(dim=24)), P.PDA_ERR_UNSUPPORTED),
    (dict(r=rotary(dim=80)), P.PDA_ERR_SHAPE), (dict(r=rotary(freq=None)), P.PDA_ERR_NULL),
    (dict(r=rotary(freq=SOME + 4)), P.PDA_ERR_ALIGNMENT), (dict(r=rotary(magnitude=float("nan"))), P.PDA_ERR_VALUE),
    (dict(r=rotary(interleaved=2)), P.PDA_ERR_VALUE), (dict(r=rotary(backward=1)), P.PDA_ERR_VALUE),
    (dict(x=P.pda_rotary_axes(5, SOME, 3)), P.PDA_ERR_UNSUPPORTED), (dict(x=P.pda_rotary_axes(0, SOME, 3)), P.PDA_ERR_SHAPE),
    (dict(x=P.pda_rotary_axes(2, SOME, 2)), P.PDA_ERR_SHAPE), (dict(x=P.pda_rotary_axes(2, None, 3)), P.PDA_ERR_NULL),
    (dict(x=P.pda_rotary_axes(2, SOME, 3), r=None), P.PDA_ERR_NULL), (dict(q=SOME + 8), P.PDA_ERR_ALIGNMENT),
    (dict(qs=255), P.PDA_ERR_SHAPE), (dict(qs=260), P.PDA_ERR_ALIGNMENT), (dict(ks=127), P.PDA_ERR_SHAPE),
    (dict(pos=None), P.PDA_ERR_NULL), (dict(q=None), P.PDA_ERR_NULL), (dict(k=None), P.PDA_ERR_NULL),
    (dict(hq=1 << 20), P.PDA_ERR_SHAPE)]


@pytest.mark.parametrize("kw,status", SHARED + [
    (dict(n=None, r=None), P.PDA_ERR_NULL), (dict(hq=0), P.PDA_ERR_SHAPE), (dict(D=520, qs=1 << 20, qos=1 << 20, ks=1 << 20, kos=1 << 20), P.PDA_ERR_UNSUPPORTED),
    (dict(dtype=2), P.PDA_ERR_UNSUPPORTED), (dict(qos=255), P.PDA_ERR_SHAPE), (dict(ko=None), P.PDA_ERR_NULL),
    (dict(qo=SOME, q=SOME, qos=264), P.PDA_ERR_SHAPE), (dict(ko=SOME, k=SOME, kos=136), P.PDA_ERR_SHAPE),
    (dict(dtype=1, qs=258, qos=256), P.PDA_ERR_ALIGNMENT), (dict(T=0, pos=None, q=None, k=None), P.PDA_OK)])
def test_norm_rotary_refuses(kw, status):
    assert call_norm(**{**dict(n=norm(), r=rotary()), **kw}) == status


def call_backward(n=None, r=None, x=None, T=3, hq=4, hkv=2, D=64, dtype=0, pos=SOME, q=SOME, qs=256, qg=SOME * 2, qgs=256,
                  dq=SOME * 3, dqs=256, k=SOME, ks=128, kg=SOME * 2, kgs=128, dk=SOME * 3, dks=128, dqw=SOME, dkw=SOME, ws=SOME,
                  size=1 << 20):
    return pda.load_library().pda_norm_rotary_backward(
        ref_of(n), ref_of(r), ref_of(x), T, hq, hkv, D, dtype, pos, q, qs, qg, qgs, dq, dqs, k, ks, kg, kgs, dk, dks, dqw, dkw,
        ws, size, None)


@pytest.mark.parametrize("kw,status", SHARED + [
    (dict(n=None), P.PDA_ERR_NULL), (dict(hq=0), P.PDA_ERR_SHAPE), (dict(dtype=2), P.PDA_ERR_UNSUPPORTED),
    (dict(qgs=255), P.PDA_ERR_SHAPE), (dict(dqs=255), P.PDA_ERR_SHAPE), (dict(kgs=127), P.PDA_ERR_SHAPE), (dict(dks=127), P.PDA_ERR_SHAPE),
    (dict(qg=None), P.PDA_ERR_NULL), (dict(dq=None), P.PDA_ERR_NULL), (dict(kg=None), P.PDA_ERR_NULL), (dict(dk=None), P.PDA_ERR_NULL),
    (dict(dq=SOME, dqs=264), P.PDA_ERR_SHAPE), (dict(dk=SOME * 2, dks=136), P.PDA_ERR_SHAPE), (dict(dqw=SOME + 4), P.PDA_ERR_ALIGNMENT),
    (dict(ws=None), P.PDA_ERR_WORKSPACE), (dict(size=100), P.PDA_ERR_WORKSPACE), (dict(ws=SOME + 4), P.PDA_ERR_ALIGNMENT),
    (dict(hkv=0), P.PDA_ERR_SHAPE), (dict(T=0, dqw=None, dkw=None, ws=None, size=0), P.PDA_OK)])
def test_backward_refuses(kw, status):
    assert call_backward(**{**dict(n=norm(), r=rotary()), **kw}) == status


def call_append(n=None, r=None, x=None, T=3, hq=4, hkv=2, D=64, blocks=9, pos=SOME, slots=SOME, q=SOME, qs=256, qo=SOME, qos=256,
                k=SOME, ks=128, v=SOME, vs=128, kc=SOME, vc=SOME):
    return pda.load_library().pda_norm_rotary_append(ref_of(n), ref_of(r), ref_of(x), T, hq, hkv, D, blocks, pos, slots, q, qs,
                                                     qo, qos, k, ks, v, vs, kc, vc, None)


@pytest.mark.parametrize("kw,status", [c for c in SHARED if c[0].get("D") != 0] + [
    (dict(D=80, qs=1024, qos=1024, ks=1024, vs=1024), P.PDA_ERR_UNSUPPORTED), (dict(hkv=0), P.PDA_ERR_SHAPE),
    (dict(blocks=0), P.PDA_ERR_SHAPE), (dict(blocks=(1 << 27) + 1), P.PDA_ERR_SHAPE), (dict(slots=None), P.PDA_ERR_NULL),
    (dict(v=None), P.PDA_ERR_NULL), (dict(kc=None), P.PDA_ERR_NULL), (dict(vc=None), P.PDA_ERR_NULL), (dict(kc=SOME + 8), P.PDA_ERR_ALIGNMENT),
    (dict(vs=127), P.PDA_ERR_SHAPE), (dict(v=SOME + 8), P.PDA_ERR_ALIGNMENT), (dict(n=None, r=rotary(backward=1)), P.PDA_ERR_VALUE),
    (dict(n=None, r=None), P.PDA_ERR_NULL), (dict(qo=None), P.PDA_ERR_NULL), (dict(T=0, pos=None, slots=None), P.PDA_OK)])
def test_append_refuses(kw, status):
    assert call_append(**{**dict(n=norm(), r=rotary()), **kw}) == status


def test_workspace_of_the_gradient():
    assert pda.pda_norm_rotary_workspace_bytes(0, 4, 2, 64) == 0
    assert 0 < pda.pda_norm_rotary_workspace_bytes(1, 4, 2, 64) < pda.pda_norm_rotary_workspace_bytes(10000, 4, 2, 64)
    assert pda.pda_norm_rotary_workspace_bytes(2 ** 31 - 1, 4, 2, 512) <= 1 << 22
    for args in ((-1, 4, 2, 64), (1, 0, 2, 64), (1, 4, -1, 64), (1, 4, 2, 12)):
        with pytest.raises(pda.PdaError):
            pda.pda_norm_rotary_workspace_bytes(*args)


def prob(**kw):
    base = dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=64, num_blocks=128, max_blocks_per_seq=17, max_context_len=257)
    base.update(kw)
    return pda.make_problem(**base)


def call_window(p=None, w=(64, 4), q=SOME, k=SOME, v=SOME, bt=SOME, lens=SOME, scale=0.125, out=SOME, ws=SOME, size=1 << 30):
    win = P.pda_window(*w) if w else None
    return pda.load_library().pda_decode_window(ref_of(p), ref_of(win), q, k, v, bt, lens, scale, out, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(p=prob(head_dim=96)), P.PDA_ERR_UNSUPPORTED), (dict(p=prob(num_q_heads=34)), P.PDA_ERR_UNSUPPORTED),
    (dict(p=prob(block_size=32)), P.PDA_ERR_UNSUPPORTED), (dict(p=prob(num_seqs=-1)), P.PDA_ERR_SHAPE),
    (dict(p=prob(max_context_len=17 * 16 + 1)), P.PDA_ERR_SHAPE), (dict(p=prob(partition_tokens=24)), P.PDA_ERR_SHAPE),
    (dict(w=None), P.PDA_ERR_NULL), (dict(w=(0, 4)), P.PDA_ERR_SHAPE), (dict(w=(-1, 4)), P.PDA_ERR_SHAPE), (dict(w=(4, -1)), P.PDA_ERR_SHAPE),
    (dict(q=None), P.PDA_ERR_NULL), (dict(k=None), P.PDA_ERR_NULL), (dict(v=None), P.PDA_ERR_NULL), (dict(bt=None), P.PDA_ERR_NULL),
    (dict(lens=None), P.PDA_ERR_NULL), (dict(out=None), P.PDA_ERR_NULL), (dict(scale=float("nan")), P.PDA_ERR_VALUE),
    (dict(q=SOME + 8), P.PDA_ERR_ALIGNMENT), (dict(out=SOME + 4), P.PDA_ERR_ALIGNMENT),
    (dict(p=prob(partition_tokens=16), ws=None, size=0), P.PDA_ERR_WORKSPACE), (dict(p=prob(partition_tokens=16), size=64), P.PDA_ERR_WORKSPACE),
    (dict(p=prob(partition_tokens=16), ws=SOME + 4), P.PDA_ERR_ALIGNMENT),
    (dict(p=prob(num_seqs=1 << 23, num_q_heads=2, num_kv_heads=2)), P.PDA_ERR_SHAPE),
    # groups of 8 tokens, launched for 8 (sequence, KV head)s: a workgroup too many
    (dict(p=prob(num_seqs=1, num_q_heads=16, num_kv_heads=1, num_query_tokens=1 << 24)), P.PDA_ERR_SHAPE),
    (dict(p=prob(num_seqs=0), q=None, k=None, v=None, bt=None, lens=None, out=None, ws=None, size=0), P.PDA_OK)])
def test_window_refuses(kw, status):
    assert call_window(**{**dict(p=prob()), **kw}) == status


def test_window_plan():
    """What is read bounds the plan, not the context."""
    p = prob(num_seqs=256, num_q_heads=32, num_kv_heads=8, head_dim=128, max_blocks_per_seq=1024, max_context_len=16384)
    plan = pda.pda_plan_window(p, 1024, 4)
    assert plan["num_partitions"] == 1 and plan["workspace_bytes"] == 0 and 1024 + 4 <= plan["partition_tokens"] <= 1024 + 64
    p.num_seqs = 8
    plan = pda.pda_plan_window(p, 4096, 16)
    assert plan["num_partitions"] == 4 and plan["workspace_bytes"] == 8 * 32 * 4 * 130 * 4
    p.partition_tokens = 48
    assert pda.pda_plan_window(p, 100, 0)["num_partitions"] == 3
    p.num_query_tokens = 64
    assert pda.pda_plan_window(p, 100, 0)["partition_tokens"] == 64


def pool(B=3, NB=9, width=4, **kw):
    a = dict(block_table=SOME, held=SOME, free_blocks=SOME, counts=SOME)
    a.update(kw)
    return P.pda_block_pool(B, NB, width, a["block_table"], a["held"], a["free_blocks"], a["counts"])


def call_resize(p, lens=SOME, rows=None, ws=SOME, size=1 << 30):
    return pda.load_library().pda_blocks_resize(ref_of(p), lens, ref_of(rows), ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(p=None), P.PDA_ERR_NULL), (dict(p=pool(B=-1)), P.PDA_ERR_SHAPE), (dict(p=pool(B=(1 << 20) + 1)), P.PDA_ERR_SHAPE),
    (dict(p=pool(NB=0)), P.PDA_ERR_SHAPE), (dict(p=pool(NB=(1 << 27) + 1)), P.PDA_ERR_SHAPE), (dict(p=pool(width=0)), P.PDA_ERR_SHAPE),
    (dict(p=pool(width=(1 << 24) + 1)), P.PDA_ERR_SHAPE), (dict(p=pool(held=None)), P.PDA_ERR_NULL), (dict(p=pool(counts=None)), P.PDA_ERR_NULL),
    (dict(p=pool(free_blocks=SOME + 2)), P.PDA_ERR_ALIGNMENT), (dict(lens=None), P.PDA_ERR_NULL), (dict(ws=None), P.PDA_ERR_WORKSPACE),
    (dict(size=8), P.PDA_ERR_WORKSPACE), (dict(ws=SOME + 4), P.PDA_ERR_ALIGNMENT),
    (dict(rows=P.pda_token_rows(-1, SOME, SOME, SOME)), P.PDA_ERR_SHAPE), (dict(rows=P.pda_token_rows(4, None, SOME, SOME)), P.PDA_ERR_SHAPE),
    (dict(rows=P.pda_token_rows(3, SOME + 2, SOME, SOME)), P.PDA_ERR_ALIGNMENT),
    (dict(p=pool(B=0, block_table=None, held=None, free_blocks=None, counts=None), lens=None, ws=None, size=0), P.PDA_OK),
    (dict(p=pool(B=0), rows=P.pda_token_rows(3, None, SOME, None)), P.PDA_ERR_SHAPE)])
def test_resize_refuses(kw, status):
    assert call_resize(**{**dict(p=pool()), **kw}) == status


@pytest.mark.parametrize("rows,table,status", [
    (None, SOME, P.PDA_ERR_NULL), (P.pda_token_rows(3, SOME, None, None), SOME, P.PDA_ERR_NULL),
    (P.pda_token_rows(3, SOME, SOME, None), None, P.PDA_ERR_NULL), (P.pda_token_rows(0, SOME, None, None), None, P.PDA_OK),
    (P.pda_token_rows(3, SOME, SOME, None), SOME + 2, P.PDA_ERR_ALIGNMENT)])
def test_slot_map_refuses(rows, table, status):
    assert pda.load_library().pda_slot_map(3, 9, 4, table, SOME, ref_of(rows), None) == status


# ---- refusals of the bindings (host tensors stand in for the GPU's) ----

@pytest.fixture
def on_device(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))


def head_args(T=5, D=64, R=64, axes=1, dtype=BF):
    q, k = torch.zeros(T, 4, D, dtype=dtype), torch.zeros(T, 2, D, dtype=dtype)
    r = pda.make_rotary(torch.ones(R // 2, dtype=torch.float64))
    n = pda.make_head_norm(torch.ones(D), torch.ones(D))
    return q, k, torch.zeros((axes, T) if axes > 1 else T, dtype=I32), r, n


def test_bindings_need_device_tensors():
    with pytest.raises(ValueError, match="device"):
        pda.make_head_norm(torch.ones(64))
    with pytest.raises(ValueError, match="device"):
        pda.new_block_pool(2, 4, 2, device="cpu")


def test_head_bindings_refuse(on_device):
    q, k, pos, r, n = head_args()
    ax = pda.make_rotary_axes(torch.zeros(32, dtype=torch.uint8), 2)
    bad = [
        (TypeError, dict(q=q.double())), (TypeError, dict(k=k.float())), (ValueError, dict(k=k[:4])), (ValueError, dict(q=q[0])),
        (TypeError, dict(positions=pos.long())), (ValueError, dict(positions=pos[:4])), (ValueError, dict(axes=ax)),
        (ValueError, dict(axes=ax, positions=torch.zeros(3, 5, dtype=I32))), (ValueError, dict(axes=ax, rotary=None, positions=torch.zeros(2, 5, dtype=I32))),
        (ValueError, dict(axes=pda.make_rotary_axes(torch.zeros(16, dtype=torch.uint8), 2), positions=torch.zeros(2, 5, dtype=I32))),
        (ValueError, dict(norm=pda.make_head_norm(torch.ones(128)))), (ValueError, dict(q_out=q[:4])), (ValueError, dict(k=None, k_out=k)),
        (ValueError, dict(q=q.transpose(0, 1).contiguous().transpose(0, 1))),
        (ValueError, dict(q=torch.zeros(5, 4, 64, dtype=BF, device="meta")))]
    for kind, kw in bad:
        args = {**dict(q=q, positions=pos, k=k, norm=n, rotary=r), **kw}
        with pytest.raises(kind):
            pda.bind_norm_rotary(**args)
    with pytest.raises(TypeError):
        pda.make_head_norm(torch.ones(64), torch.ones(64, dtype=BF))
    with pytest.raises(TypeError):
        pda.make_rotary_axes(torch.zeros(32, dtype=I32), 2)
    g, gk = torch.zeros_like(q), torch.zeros_like(k)
    for kw in (dict(norm=None), dict(k_grad=None), dict(k=None), dict(q_grad=g[:4]), dict(dq=g[:, :2]), dict(dq_weight=torch.zeros(32)),
               dict(workspace=torch.zeros(1 << 12, 2, dtype=torch.uint8)[:, 0])):
        args = {**dict(q=q, q_grad=g, positions=pos, k=k, k_grad=gk, norm=n, rotary=r), **kw}
        with pytest.raises(ValueError):
            pda.bind_norm_rotary_backward(**args)
    with pytest.raises(TypeError):
        pda.bind_norm_rotary_backward(q, g.float(), pos, k, gk, norm=n, rotary=r)
    kc, vc, slots = torch.zeros(9, 2, 8, 16, 8, dtype=BF), torch.zeros(9, 2, 16, 64, dtype=BF), torch.zeros(5, dtype=I32)
    for kind, kw in ((ValueError, dict(kc=kc[:, :, :4])), (ValueError, dict(vc=vc[:, :1])), (TypeError, dict(slots=slots.long())),
                     (ValueError, dict(slots=slots[:3])), (ValueError, dict(v=k[:, :1])), (ValueError, dict(q=None, q_out=q)),
                     (ValueError, dict(norm=None, rotary=None)), (TypeError, dict(kc=kc.float())), (ValueError, dict(q=q[:4]))):
        args = {**dict(q=q, k=k, v=k, positions=pos, slots=slots, kc=kc, vc=vc, norm=n, rotary=r), **kw}
        with pytest.raises(kind):
            pda.bind_norm_rotary_append(args["q"], args["k"], args["v"], args["positions"], args["slots"], args["kc"], args["vc"],
                                        args["norm"], args["rotary"], q_out=args.get("q_out"))


def test_window_binding_refuses(on_device):
    q, kc, vc = torch.zeros(3, 4, 64, dtype=BF), torch.zeros(9, 2, 8, 16, 8, dtype=BF), torch.zeros(9, 2, 16, 64, dtype=BF)
    bt, lens = torch.zeros(3, 4, dtype=I32), torch.zeros(3, dtype=I32)
    for kind, kw in ((ValueError, dict(max_context_len=None)), (pda.PdaError, dict(window=0)), (pda.PdaError, dict(sinks=-1)),
                     (pda.PdaError, dict(max_context_len=65)), (ValueError, dict(q=q[:2])), (TypeError, dict(q=q.float())),
                     (ValueError, dict(lens=lens[:2])), (ValueError, dict(q=torch.zeros(3, 0, 4, 64, dtype=BF))),
                     (ValueError, dict(out=torch.zeros(3, 4, 32))), (ValueError, dict(vc=vc[:8])),
                     (ValueError, dict(workspace=torch.zeros(64, 2, dtype=torch.uint8)[:, 0]))):
        a = {**dict(q=q, kc=kc, vc=vc, bt=bt, lens=lens, out=None, window=8, sinks=0, max_context_len=64, workspace=None), **kw}
        with pytest.raises(kind):
            pda.bind_decode_window(a["q"], a["kc"], a["vc"], a["bt"], a["lens"], 0.125, a["out"], window=a["window"], sinks=a["sinks"],
                                   max_context_len=a["max_context_len"], workspace=a["workspace"])


def test_block_bindings_refuse(on_device):
    i = lambda *s: torch.zeros(s, dtype=I32)
    p = pda.make_block_pool(i(3, 4), i(3), i(9), i(2))
    for kind, args in ((ValueError, (i(3), i(3), i(9), i(2))), (ValueError, (i(3, 4), i(2), i(9), i(2))), (ValueError, (i(3, 4), i(3), i(9), i(3))),
                       (TypeError, (i(3, 4).long(), i(3), i(9), i(2))), (ValueError, (i(4, 3).t(), i(3), i(9), i(2)))):
        with pytest.raises(kind):
            pda.make_block_pool(*args)
    for kind, args, kw in ((ValueError, (i(2),), {}), (TypeError, (i(3).long(),), {}), (ValueError, (i(3),), dict(row_start=i(4))),
                           (ValueError, (i(3),), dict(row_start=i(3), slots=i(6))), (ValueError, (i(3),), dict(positions=i(5), slots=i(6))),
                           (TypeError, (i(3),), dict(slots=i(6).long()))):
        with pytest.raises(kind):
            pda.bind_blocks_resize(p, *args, **kw)
    with pytest.raises(ValueError):
        pda.bind_slot_map(i(3, 4), i(3), 9)
    with pytest.raises(ValueError):
        pda.bind_slot_map(i(3), i(3), 9, slots=i(3))


# ---- the memory of calls on a given stream ----

from test_streams_host import Recorder, Stream, bf16_inputs, given  # noqa: E402,F401


@pytest.mark.parametrize("which", ["bind", "pda"])
def test_memory_of_a_given_stream(monkeypatch, given, which):  # noqa: F811
    rec = Recorder(monkeypatch)
    q, k, pos, r, n = head_args()

    def call(name, *args, **kw):
        got = getattr(pda, f"{which}_{name}")(*args, stream=given, **kw)
        return got.result if which == "bind" else got

    rec.check(call("norm_rotary", q, pos, k, n, r), cleared=True)
    dq, dk, dqw, dkw = call("norm_rotary_backward", q, q, pos, k, k, n, r)
    rec.check([dq, dk], cleared=True)
    rec.check([dqw, dkw], cleared=False)
    qw, kc, vc, table, lens = bf16_inputs()
    rec.check([call("norm_rotary_append", q, k, k, pos, torch.zeros(5, dtype=I32), kc, vc, n, r)], cleared=True)
    rec.check([call("decode_window", qw, kc, vc, table, lens, 0.125, window=40, max_context_len=64, partition_tokens=16)], cleared=False)
    i = lambda *s: torch.zeros(s, dtype=I32)
    before = len(rec.made)
    call("blocks_resize", pda.make_block_pool(i(3, 4), i(3), i(9), i(2)), i(3))
    assert len(rec.made) == before + 1  # its workspace, cleared on the call's stream
    stream, workspace = list(rec.made.values())[-1]
    assert rec.cleared[id(workspace)] == stream
