"""Rotary positions against complex rotations in 64 bits, through the C ABI.

Tolerance: one rounding of the result (half a step of its type) and, of fp32, the cosine and sine (within
2 steps of 2^-24, of an angle rounded once: pi 2^-24 off), two products and a sum: 8 * 2^-24 of |a| + |b|."""
import math

import pytest
import torch

from seq_util import DTYPES, assert_within, half_step

pytestmark = pytest.mark.gpu


def turned(x, positions, turns, rotary, half, factor, sign):
    z = torch.polar(torch.tensor(factor, dtype=torch.float64), 2 * math.pi * sign * positions.double()[:, None] * turns)[:, None]
    x = x.double()
    at = (slice(0, rotary // 2), slice(rotary // 2, rotary)) if half else (slice(0, rotary, 2), slice(1, rotary, 2))
    y, size = x.clone(), torch.zeros_like(x)
    w = torch.complex(x[..., at[0]], x[..., at[1]]) * z
    y[..., at[0]], y[..., at[1]] = w.real, w.imag
    size[..., at[0]] = size[..., at[1]] = factor * (x[..., at[0]].abs() + x[..., at[1]].abs())
    return y, size


@pytest.mark.parametrize("half", [True, False], ids=["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,dim,rotary,far", [(1, 1, 2, 2, 10), (5, 3, 32, 32, 4096), (16, 40, 128, 128, 131072), (33, 7, 80, 40, 50),
                                                       (3, 2, 64, 12, 2 ** 31 - 1), (100, 5, 10, 6, 1000), (257, 24, 128, 64, 8191),
                                                       (2, 1, 1024, 1024, 99), (700, 3, 6, 2, 77)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_both_directions(dnb, dtype, rows, heads, dim, rotary, far, half):
    dt = DTYPES[dtype]
    gen = torch.Generator().manual_seed(rows + dim)
    x = torch.randn(rows, heads, dim, generator=gen).to(dt)
    pos = torch.randint(0, far, (rows,), generator=gen, dtype=torch.int32)
    pos[0] = far - 1
    if rows > 2:
        pos[1], pos[2] = 0, -far
    turns = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary) / (2 * math.pi)
    order, code = (dnb.DNB_ROPE_HALF if half else dnb.DNB_ROPE_INTERLEAVED), dnb.DNB_F32 if dtype == "f32" else dnb.DNB_BF16
    for call, sign in ((dnb.dnb_op_rope_forward, 1.0), (dnb.dnb_op_rope_backward, -1.0)):
        y = torch.full(x.shape, float("nan"), dtype=dt, device="cuda")
        xd, pd, td = x.cuda(), pos.cuda(), turns.cuda()
        call(xd, pd, td, y, rows, heads, dim, rotary, order, 1.25, code)
        want, size = turned(x, pos, turns, rotary, half, 1.25, sign)
        tol = 8 * 2.0 ** -24 * size + (half_step(dt) * want.abs() if dtype == "bf16" else 0)
        # far - 1 in 64 bits: the product itself is off by 2^-53 of some turns
        tol = tol + 2 * math.pi * far * 2.0 ** -52 * size
        assert_within(y, want, tol, "y")
        call(xd, pd, td, xd, rows, heads, dim, rotary, order, 1.25, code)   # in place
        assert torch.equal(xd, y)


def test_some_heads_of_wider_rows(dnb):
    """Queries and keys of a row that also holds values, in place; the values stay."""
    rows, heads, dim = 37, 6, 64
    wide = torch.randn(rows, (heads + 3) * dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    pos = torch.arange(rows, dtype=torch.int32) * 100
    turns = 500.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    w = wide.cuda()
    dnb.dnb_op_rope_forward(w, pos.cuda(), turns.cuda(), w, rows, heads, dim, dim, dnb.DNB_ROPE_HALF, x_stride=w.shape[1], y_stride=w.shape[1])
    want, size = turned(wide[:, :heads * dim].reshape(rows, heads, dim), pos, turns, dim, True, 1.0, 1.0)
    assert_within(w[:, :heads * dim].reshape(rows, heads, dim), want, 8 * 2.0 ** -24 * size + half_step(torch.bfloat16) * want.abs(), "turned")
    assert torch.equal(w[:, heads * dim:].cpu(), wide[:, heads * dim:])


def test_backward_is_the_adjoint(dnb):
    """<forward(x), dy> = <x, backward(dy)>, and differences of a linear map are the map itself."""
    rows, heads, dim = 50, 4, 48
    gen = torch.Generator().manual_seed(2)
    x, dy = (torch.randn(rows, heads, dim, generator=gen).cuda() for _ in range(2))
    pos = torch.randint(0, 9999, (rows,), generator=gen, dtype=torch.int32).cuda()
    turns = torch.rand(12, generator=gen, dtype=torch.float64).cuda()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dnb.dnb_op_rope_forward(x, pos, turns, y, rows, heads, dim, 24, dnb.DNB_ROPE_INTERLEAVED, 0.7, dnb.DNB_F32)
    dnb.dnb_op_rope_backward(dy, pos, turns, dx, rows, heads, dim, 24, dnb.DNB_ROPE_INTERLEAVED, 0.7, dnb.DNB_F32)
    a, b = (y.double() * dy.double()).sum(), (x.double() * dx.double()).sum()
    assert abs(float(a - b)) <= 8 * 2.0 ** -24 * 2 * float((x.double().abs() * dy.double().abs()).sum() + (dx.double().abs() * x.double().abs()).sum())
