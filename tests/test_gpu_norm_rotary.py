"""Head norms, rotary positions with several axes, their gradients and the append through a slot
map, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2405_11143_amd as pda
from more_reference import HEAD_UNITS, HALF_STEP, cache_of, head_grad, head_tolerance, normed, turned

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


class Case:
    """Inputs of one call: rows of a fused projection, positions on `axes` axes with padding."""

    def __init__(self, T, Hq, Hkv, D, R, dtype=BF, axes=1, interleaved=False, norm=True, weights=True, offset=0.0,
                 weight_dtype=None, magnitude=1.0, seed=0, padding=True, far=100000, eps=1e-6):
        gen = torch.Generator().manual_seed(seed + T + D + R)
        self.T, self.Hq, self.Hkv, self.D, self.R, self.dtype = T, Hq, Hkv, D, R, dtype
        self.axes, self.interleaved, self.offset, self.magnitude, self.eps = axes, interleaved, offset, magnitude, eps
        size = torch.exp2(torch.randn((T, 1, 1), generator=gen) * 3)
        self.rows = (torch.randn((T, Hq + 2 * Hkv + 1, D), generator=gen) * size).to(dtype).cuda()
        self.q, self.k = self.rows[:, :Hq], self.rows[:, Hq:Hq + Hkv] if Hkv else None
        self.v = self.rows[:, Hq + Hkv:Hq + 2 * Hkv]
        self.positions = torch.randint(0, far, (axes, T), generator=gen, dtype=torch.int32)
        if axes > 1:
            self.positions[1:] -= far // 2  # (further axes may be negative)
        if padding and T > 2:
            self.positions[0, torch.rand(T, generator=gen) < 0.2] = -1
        self.positions = self.positions.cuda()
        self.real = self.positions[0] >= 0
        self.inv_freq = (10000.0 ** (-2.0 * torch.arange(R // 2, dtype=torch.float64) / R)).cuda() if R else None
        self.axis = torch.randint(0, axes, (R // 2,), generator=gen).to(torch.uint8).cuda()
        wt = weight_dtype or dtype
        w = lambda: (1 - offset + 0.3 * torch.randn(D, generator=gen)).to(wt).cuda() if weights else None
        self.qw, self.kw = w(), w()
        self.norm = pda.make_head_norm(self.qw, self.kw, eps=eps, weight_offset=offset) if norm else None
        self.rotary = pda.make_rotary(self.inv_freq, interleaved=interleaved, magnitude=magnitude) if R else None
        self.axes_arg = pda.make_rotary_axes(self.axis, axes) if R and axes > 1 else None
        self.pos_arg = self.positions if self.axes_arg is not None else self.positions[0]
        self.kw_args = dict(norm=self.norm, rotary=self.rotary, axes=self.axes_arg)

    def exact(self, rows, weight, sign=1.0):
        """(y, tolerance) of rows."""
        z = rows.double()
        if self.norm is not None:
            z = normed(z, weight, self.eps, self.offset)
        y, size = (z, z.abs()) if self.inv_freq is None else turned(z, self.positions, self.inv_freq, self.axis,
                                                                    self.interleaved, sign, self.magnitude)
        return y, head_tolerance(y, size, self.dtype)


def assert_rows(got, want, tol, real):
    assert torch.isfinite(got[real].float()).all()
    worst = ((got.double() - want).abs() / tol.clamp(min=1e-300))[real].max() if real.any() else 0.0
    assert float(worst) <= 1.0, float(worst)


SHAPES = [  # T, Hq, Hkv, D, R
    (1, 1, 0, 64, 64), (1, 8, 2, 128, 128), (7, 28, 4, 128, 64), (33, 16, 16, 80, 80), (65, 5, 3, 80, 48), (3, 2, 1, 8, 0),
    (130, 32, 8, 128, 128), (19, 16, 4, 256, 256), (5, 3, 2, 512, 496), (11, 4, 1, 24, 16), (2500, 3, 1, 128, 128),
    (40, 300, 20, 64, 32)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kw", [dict(), dict(axes=3, interleaved=True, weight_dtype=F32, offset=1.0),
                                dict(norm=False, axes=4), dict(weights=False, magnitude=1.25, axes=2)])
def test_forward(shape, dtype, kw):
    if shape[4] == 0 and not kw.get("norm", True):
        pytest.skip("nothing to do")
    if dtype == F32 and kw.get("weight_dtype") == F32:
        kw = dict(kw, weight_dtype=BF)
    c = Case(*shape, dtype=dtype, **kw)
    q_out = torch.full((c.T, c.Hq, c.D), 7.0, dtype=dtype, device="cuda")
    k_out = torch.full((c.T, c.Hkv, c.D), 7.0, dtype=dtype, device="cuda") if c.Hkv else None
    before = c.rows.clone()
    pda.pda_norm_rotary(c.q, c.pos_arg, c.k, q_out=q_out, k_out=k_out, **c.kw_args)
    assert torch.equal(c.rows, before)
    assert_rows(q_out, *c.exact(c.q, c.qw), c.real)
    assert (q_out[~c.real] == 7.0).all()  # padding is left as it was
    if c.Hkv:
        assert_rows(k_out, *c.exact(c.k, c.kw), c.real)
        assert (k_out[~c.real] == 7.0).all()


def test_turning_back_is_the_inverse_and_the_gradient():
    c = Case(77, 6, 2, 128, 96, dtype=F32, norm=False, axes=3)
    back = pda.make_rotary(c.inv_freq, backward=True)
    q1, k1 = pda.pda_norm_rotary(c.q, c.pos_arg, c.k, rotary=c.rotary, axes=c.axes_arg)
    q2, _ = pda.pda_norm_rotary(q1, c.pos_arg, k1, rotary=back, axes=c.axes_arg)
    tol = 2 * HEAD_UNITS * 2.0 ** -24 * 2 * c.q.abs().amax(-1, keepdim=True)
    assert ((q2 - c.q).abs() <= tol)[c.real].all()
    y, size = turned(q1.double(), c.positions, c.inv_freq, c.axis, False, -1.0)
    assert_rows(q2, y, head_tolerance(y, size, F32), c.real)


def test_one_axis_is_the_plain_rotation():
    """Axes that all say the same give one axis's bits, and both what pda_rotary_apply gives: not its
    bits, since either product of x cos a - y sin a may be the one that a multiply-add
    leaves unrounded, but each call is within head_tolerance of the exact value, so the two are
    within twice that of each other."""
    c = Case(64, 8, 2, 128, 128, norm=False)
    want = pda.pda_rotary_apply(c.q, c.positions[0], c.rotary, c.k)
    got = pda.pda_norm_rotary(c.q, c.positions[0], c.k, rotary=c.rotary)
    same = pda.pda_norm_rotary(c.q, c.positions.repeat(3, 1), c.k, rotary=c.rotary,
                               axes=pda.make_rotary_axes(torch.arange(64, dtype=torch.uint8, device="cuda") % 3, 3))
    for x, y, z, rows in zip(want, got, same, (c.q, c.k)):
        assert torch.equal(y, z)
        assert ((x.double() - y.double()).abs() <= 2 * c.exact(rows, None)[1])[c.real].all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place_and_strides(dtype):
    """Rows where they lie in the fused projection, in place; the values between them stay."""
    c = Case(50, 8, 2, 128, 128, dtype=dtype)
    want = pda.pda_norm_rotary(c.q, c.pos_arg, c.k, **c.kw_args)
    rows = c.rows.clone()
    q, k = rows[:, :8], rows[:, 8:10]
    pda.pda_norm_rotary(q, c.pos_arg, k, q_out=q, k_out=k, **c.kw_args)
    for got, x, before in ((q, want[0], c.q), (k, want[1], c.k)):
        assert torch.equal(got[c.real], x[c.real]) and torch.equal(got[~c.real], before[~c.real])
    assert torch.equal(rows[:, 10:], c.rows[:, 10:])
    two = pda.make_rotary_axes(torch.zeros(64, dtype=torch.uint8, device="cuda"), 2)
    wide = torch.zeros((2, 90), dtype=torch.int32, device="cuda")  # (a row stride past T)
    wide[:, :50] = c.positions
    got = pda.pda_norm_rotary(c.q, wide[:, :50], c.k, norm=c.norm, rotary=c.rotary, axes=two)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_odd_rows_stay_by_themselves():
    """Rows of zeros, NaN and infinities: no other row changes."""
    c = Case(20, 4, 2, 128, 128, padding=False)
    want = pda.pda_norm_rotary(c.q, c.pos_arg, c.k, **c.kw_args)
    rows = c.rows.clone()
    rows[3, 1], rows[4, 4, 7], rows[5, 0, 9] = 0.0, float("nan"), float("inf")
    got = pda.pda_norm_rotary(rows[:, :4], c.pos_arg, rows[:, 4:6], **c.kw_args)
    assert (got[0][3, 1] == 0).all() and torch.isnan(got[1][4, 0]).any() and not torch.isfinite(got[0][5, 0]).all()
    same = torch.ones((20, 4), dtype=torch.bool, device="cuda")
    same[3, 1] = same[5, 0] = False
    assert torch.equal(got[0][same], want[0][same])
    assert torch.equal(got[1][4, 1], want[1][4, 1])


# ------------------------------------------------------------------- gradient --

@pytest.mark.parametrize("shape", [s for s in SHAPES] + [(3000, 12, 2, 64, 64)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kw", [dict(), dict(axes=3, interleaved=True, weight_dtype=F32, offset=1.0),
                                dict(weights=False, magnitude=1.25)])
def test_backward(shape, dtype, kw):
    c = Case(*shape, dtype=dtype, **kw)
    gen = torch.Generator().manual_seed(5)
    grads = [torch.randn((c.T, h, c.D), generator=gen).to(dtype).cuda() if h else None for h in (c.Hq, c.Hkv)]
    dq, dk = (torch.full((c.T, h, c.D), 7.0, dtype=dtype, device="cuda") if h else None for h in (c.Hq, c.Hkv))
    dqw, dkw = (torch.full((c.D,), 7.0, device="cuda") if h else None for h in (c.Hq, c.Hkv))
    pda.pda_norm_rotary_backward(c.q, grads[0], c.pos_arg, c.k, grads[1], dq=dq, dk=dk, dq_weight=dqw, dk_weight=dkw,
                                 **c.kw_args)
    for x, g, w, dx, dw in ((c.q, grads[0], c.qw, dq, dqw), (c.k, grads[1], c.kw, dk, dkw)):
        if x is None:
            continue
        want, scale, hu, hu_size = head_grad(x.double(), g.double(), w, c.eps, c.offset, c.positions, c.inv_freq, c.axis,
                                             c.interleaved, c.magnitude)
        # (the formula's two sums count as one each beside the row's own)
        tol = HALF_STEP[dtype] * want.abs() + 2 * HEAD_UNITS * 2.0 ** -24 * scale * (1 + HALF_STEP[dtype])
        assert_rows(dx, want, tol, c.real)
        assert (dx[~c.real] == 7.0).all()
        # a weight's sum: a thread's own rows, then 6 + 4 levels, then a run of partial sums and 32 runs
        terms = -(-c.T // 1024) * (c.Hq + c.Hkv) + 10 + min(c.T, 1024) / 32 + 32
        allowed = (HEAD_UNITS + terms) * 2.0 ** -24 * hu_size[c.real].sum((0, 1))
        assert ((dw.double() - hu[c.real].sum((0, 1))).abs() <= allowed + 1e-300).all()


def test_backward_against_differences():
    """The gradient of sum(y * g), y from the forward call, by central differences in fp32."""
    c = Case(3, 2, 1, 64, 32, dtype=F32, axes=2, offset=1.0, seed=4, padding=False, far=50)
    x0 = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(1)).cuda()
    k0 = torch.randn((3, 1, 64), generator=torch.Generator().manual_seed(2)).cuda()
    g, gk = torch.randn_like(x0), torch.randn_like(k0)

    def loss(x, k, norm):
        y, z = pda.pda_norm_rotary(x, c.pos_arg, k, norm=norm, rotary=c.rotary, axes=c.axes_arg)
        return float((y.double() * g).sum() + (z.double() * gk).sum())

    dq, dk, dqw, dkw = pda.pda_norm_rotary_backward(x0, g, c.pos_arg, k0, gk, **c.kw_args)
    h = 2.0 ** -6  # (third derivatives h^2 = 2^-12, roundings 2^-24 / h per element of a loss of about 100 terms of size 1)
    for t, grad in ((x0, dq), (k0, dk)):
        for at in ((0, 0, 0), (1, 0, 33), (2, 0, 63), (1, 0, 5)):
            hi, lo = t.clone(), t.clone()
            hi[at] += h
            lo[at] -= h
            d = (loss(hi if t is x0 else x0, hi if t is k0 else k0, c.norm) -
                 loss(lo if t is x0 else x0, lo if t is k0 else k0, c.norm)) / (2 * h)
            assert abs(d - float(grad[at])) <= 4e-3, (at, d, float(grad[at]))
    for w, grad, which in ((c.qw, dqw, 0), (c.kw, dkw, 1)):
        for i in (0, 31, 63):
            ws = []
            for s in (h, -h):
                w2 = w.clone()
                w2[i] += s
                ws.append(pda.make_head_norm(w2 if which == 0 else c.qw, w2 if which else c.kw, eps=c.eps, weight_offset=1.0))
            d = (loss(x0, k0, ws[0]) - loss(x0, k0, ws[1])) / (2 * h)
            assert abs(d - float(grad[i])) <= 4e-3  # (linear in the weight)


def test_backward_in_place_reproducible_and_only_some():
    c = Case(700, 12, 2, 128, 128)
    g, gk = torch.randn_like(c.q.contiguous()), torch.randn_like(c.k.contiguous())
    first = pda.pda_norm_rotary_backward(c.q, g, c.pos_arg, c.k, gk, **c.kw_args)
    again = pda.pda_norm_rotary_backward(c.q, g, c.pos_arg, c.k, gk, **c.kw_args)
    for x, y in zip(first, again):
        assert torch.equal(x, y)
    g2, gk2 = g.clone(), gk.clone()
    dq, dk, dqw, dkw = pda.pda_norm_rotary_backward(c.q, g2, c.pos_arg, c.k, gk2, dq=g2, dk=gk2, **c.kw_args)
    assert dq is g2 and torch.equal(g2[c.real], first[0][c.real]) and torch.equal(gk2[c.real], first[1][c.real])
    assert torch.equal(g2[~c.real], g[~c.real]) and torch.equal(dqw, first[2]) and torch.equal(dkw, first[3])
    rows = c.rows.clone()  # the gradient over the fused rows themselves
    q, k = rows[:, :12], rows[:, 12:14]
    pda.pda_norm_rotary_backward(q, g, c.pos_arg, k, gk, dq=q, dk=k, **c.kw_args)
    assert torch.equal(q[c.real], first[0][c.real]) and torch.equal(rows[:, 14:], c.rows[:, 14:])
    only_q = pda.pda_norm_rotary_backward(c.q, g, c.pos_arg, norm=c.norm, rotary=c.rotary)
    assert torch.equal(only_q[0], first[0]) and torch.equal(only_q[2], first[2]) and only_q[1] is only_q[3] is None


def test_no_tokens_and_padding_alone():
    empty = Case(0, 4, 2, 128, 128)
    _, _, dqw, dkw = pda.pda_norm_rotary_backward(empty.q, empty.q, empty.pos_arg, empty.k, empty.k, **empty.kw_args)
    assert (dqw == 0).all() and (dkw == 0).all()
    pda.pda_norm_rotary(empty.q, empty.pos_arg, empty.k, **empty.kw_args)
    c = Case(9, 4, 2, 128, 128)
    c.positions.fill_(-1)
    dq, dk, dqw, dkw = pda.pda_norm_rotary_backward(c.q, c.q, c.pos_arg, c.k, c.k, **c.kw_args)
    for x in (dq, dk, dqw, dkw):
        assert (x == 0).all()


def test_backward_captured():
    """The gradient captured into a graph and replayed with other contents."""
    c = Case(300, 8, 2, 128, 128)
    g, gk = torch.randn_like(c.q.contiguous()), torch.randn_like(c.k.contiguous())
    stream = torch.cuda.Stream()
    call = pda.bind_norm_rotary_backward(c.q, g, c.pos_arg, c.k, gk, stream=stream, **c.kw_args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for _ in range(3):
        g.normal_()
        c.rows.mul_(1.5)
        for t in call.result:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(call.result, pda.pda_norm_rotary_backward(c.q, g, c.pos_arg, c.k, gk, **c.kw_args)):
            assert torch.equal(x, y)


# --------------------------------------------------------------------- append --

@pytest.mark.parametrize("T,Hq,Hkv,D,R", [(1, 8, 2, 64, 64), (5, 32, 8, 128, 128), (300, 28, 4, 128, 64), (2200, 6, 2, 64, 32),
                                          (2100, 8, 1, 128, 128)])
@pytest.mark.parametrize("kw", [dict(), dict(axes=3, interleaved=True, offset=1.0), dict(norm=False)])
def test_append(T, Hq, Hkv, D, R, kw):
    c = Case(T, Hq, Hkv, D, R, **kw)
    rng = np.random.RandomState(T)
    NB = T // 10 + 4
    slots = torch.from_numpy(rng.permutation(16 * NB)[:T].astype(np.int32))
    if T > 4:
        slots[1], slots[2], slots[3] = -1, 16 * NB, 2 ** 31 - 1  # nothing is stored
    slots = slots.cuda()
    k_rows, v_rows = (torch.randn((NB, Hkv, 16, D), device="cuda").to(BF) for _ in range(2))
    kc, vc = cache_of(k_rows, v_rows)
    vc = vc.clone()
    q_out = torch.full((T, Hq, D), 7.0, dtype=BF, device="cuda")
    pda.pda_norm_rotary_append(c.q, c.k, c.v, c.pos_arg, slots, kc, vc, q_out=q_out, **c.kw_args)
    assert_rows(q_out, *c.exact(c.q, c.qw), c.real)
    assert (q_out[~c.real] == 7.0).all()
    r = torch.nonzero(c.real & (slots >= 0) & (slots < 16 * NB))[:, 0]
    page, place = slots[r].long() // 16, slots[r].long() % 16
    got = kc.transpose(2, 3).reshape(NB, Hkv, 16, D)
    y, tol = c.exact(c.k, c.kw)
    assert_rows(got[page, :, place], y[r], tol[r], torch.ones(len(r), dtype=torch.bool, device="cuda"))
    v_rows[page, :, place] = c.v[r]
    assert torch.equal(vc, v_rows)
    k_rows[page, :, place] = got[page, :, place]
    assert torch.equal(got, k_rows)  # nothing else changed


def test_append_of_rows_as_they_are():
    c = Case(40, 2, 2, 128, 128, padding=False)
    kc, vc = cache_of(*(torch.zeros((5, 2, 16, 128), dtype=BF, device="cuda") for _ in range(2)))
    slots = torch.randperm(80, dtype=torch.int32, device="cuda")[:40].contiguous()
    assert pda.pda_norm_rotary_append(None, c.k, c.v, c.pos_arg, slots, kc, vc) is None
    at = slots.long()
    assert torch.equal(kc.transpose(2, 3).reshape(5, 2, 16, 128)[at // 16, :, at % 16], c.k)
    assert torch.equal(vc[at // 16, :, at % 16], c.v)
