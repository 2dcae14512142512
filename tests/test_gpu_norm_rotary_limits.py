"""The limits that include/pda_norm_rotary.h states, against 64 bits: the largest and smallest elements of
a norm, the smallest eps, and positions to the end of 32 bits."""
import pytest
import torch

import paper_2405_11143_amd as pda
from more_reference import HALF_STEP, HEAD_UNITS, head_grad, head_tolerance, normed, turned
from test_gpu_norm_rotary import assert_rows

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows_of(D, eps, dtype):
    """Rows [T, 3, D] whose largest elements are near the limits for eps: all of a size, and one beside zeros."""
    gen = torch.Generator().manual_seed(D)
    sizes = [58.0, 30.0, 0.0, -58.5] if eps < 2.0 ** -118 else [58.0, -50.0, -58.5, -60.0, -64.0, -75.0]
    x = torch.randn((2 * len(sizes), 3, D), generator=gen, dtype=torch.float64)
    x /= x.abs().amax(-1, keepdim=True)
    x[1::2] = torch.where(x[1::2].abs() == 1, x[1::2], 0.0)
    x *= torch.exp2(torch.tensor(sizes, dtype=torch.float64)).repeat_interleave(2)[:, None, None]
    if eps > 0:
        x[-1] = 0.0
    return x.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 64, 512])
@pytest.mark.parametrize("eps", [0.0, 1e-42, 2.0 ** -118])
def test_sizes_of_elements(D, eps, dtype):
    x = rows_of(D, eps, dtype)
    q, k = x[:, :2], x[:, 2:]
    w = (1 + 0.3 * torch.randn(D, generator=torch.Generator().manual_seed(1))).to(dtype).cuda()
    norm = pda.make_head_norm(w, w, eps=eps)
    positions = torch.zeros(x.shape[0], dtype=torch.int32, device="cuda")
    real = positions == 0
    held = torch.tensor(eps, dtype=F32).item()  # eps as the library gets it
    g = torch.randn(x.shape, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    got = pda.pda_norm_rotary(q, positions, k, norm=norm)
    for y, rows in zip(got, (q, k)):
        want = normed(rows.double(), w, held)
        assert_rows(y, want, head_tolerance(want, want.abs(), dtype) + 2.0 ** -133, real)
    grads = pda.pda_norm_rotary_backward(q, g[:, :2], positions, k, g[:, 2:], norm=norm)
    for dx, rows, gr in zip(grads, (q, k), (g[:, :2], g[:, 2:])):
        want, scale, _, _ = head_grad(rows.double(), gr.double(), w, held, 0.0, None, None, None, False)
        tol = HALF_STEP[dtype] * want.abs() + 2 * HEAD_UNITS * 2.0 ** -24 * scale * (1 + HALF_STEP[dtype])
        assert_rows(dx, want, tol + 2.0 ** -133, real)


def test_positions_to_the_end_of_32_bits():
    """An angle's error does not grow with the position."""
    gen = torch.Generator().manual_seed(5)
    positions = torch.tensor([[0, 1, 2 ** 31 - 1, 2 ** 30 + 12345, 10 ** 6 + 3], [-2 ** 31, 2 ** 31 - 1, -1, -2 ** 30 - 777, 5]],
                             dtype=torch.int32, device="cuda")
    q = torch.randn((5, 3, 64), generator=gen).cuda()
    f = 10000.0 ** (-2.0 * torch.arange(32, dtype=torch.float64) / 64)
    axis = (torch.arange(32) % 2).to(torch.uint8).cuda()
    got, _ = pda.pda_norm_rotary(q, positions, rotary=pda.make_rotary(f.cuda()), axes=pda.make_rotary_axes(axis, 2))
    y, size = turned(q.double(), positions, f.cuda(), axis, False)
    # (angles of up to 2^31, in 64 bits, on either side)
    assert_rows(got, y, head_tolerance(y, size, F32) + 2.0 ** 31 * 2.0 ** -51 * size, positions[0] >= 0)
