"""The paged cache's kernels where offsets are not what they should be, and where there are more workgroups than one dimension of a launch
takes."""
import math

import pytest
import torch

from paged_util import Cache, ints
from seq_util import DTYPES

pytestmark = pytest.mark.gpu
GUARD = 4096   # values before and behind a tensor


def guarded(shape, dtype, fill):
    """A tensor in the middle of memory that holds `fill`."""
    n = math.prod(shape)
    around = torch.full((n + 2 * GUARD,), fill, dtype=dtype, device="cuda")
    return around[GUARD:GUARD + n].view(shape), around


def untouched(around, fill):
    return bool((around[:GUARD] == fill).all() and (around[-GUARD:] == fill).all())


OFFSETS = [[0, 7, 3, 12], [12, 8, 4, 0], [5, 12, 0, 12], [0, 12, 0, 12], [-9, 30, -2 ** 31, 2 ** 31 - 1], [2 ** 31 - 1, 0, 0, 0]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("qo", OFFSETS)
def test_offsets_that_decrease(dnb, dtype, qo):
    """Which of two sequences a row is of is not defined then; nothing outside the tensors is written."""
    heads, kv, dim, rows, dt = 4, 2, 64, 12, DTYPES[dtype]
    cache = Cache([40, 3, 150], 16, kv, dim, dt)
    layout = cache.layout_of(dnb)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(rows, (heads + 2 * kv) * dim, generator=gen).to(dt).cuda()
    q, k, v = x.split([heads * dim, kv * dim, kv * dim], 1)
    pools = []
    for t in cache.to_gpu():
        pool, around = guarded(t.shape, dt, 3.0)
        pool.copy_(torch.nan_to_num(t))
        pools.append((pool, around))
    out, out_around = guarded((rows, heads, dim), dt, 5.0)
    q_out, q_around = guarded((rows, heads, dim), dt, 5.0)
    lse, lse_around = guarded((heads, rows), torch.float32, 5.0)
    turns = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).cuda()
    offs, lens, table = ints(qo), ints(cache.lengths), ints(cache.table)
    qk = dnb.dnb_qk_layout(rows, heads, kv, dim, dim, dtype=layout.dtype, q_stride=x.shape[1], k_stride=x.shape[1], v_stride=x.shape[1])
    dnb.dnb_op_paged_append(qk, layout, q, k, v, None, None, None, turns, offs, lens, table, q_out, pools[0][0], pools[1][0])
    plan = dnb.dnb_paged_attn_create(layout, heads, rows)
    ws, ws_around = guarded((dnb.dnb_paged_attn_workspace_bytes(plan),), torch.uint8, 0xa5)
    dnb.dnb_paged_attn_forward(plan, q_out, pools[0][0], pools[1][0], offs, lens, table, out, lse, ws)
    torch.cuda.synchronize()
    dnb.dnb_paged_attn_destroy(plan)
    for around, fill in ((pools[0][1], 3.0), (pools[1][1], 3.0), (out_around, 5.0), (q_around, 5.0), (lse_around, 5.0), (ws_around, 0xa5)):
        assert untouched(around, fill)


def test_rotation_of_more_rows_than_2_22_workgroups(dnb):
    """A workgroup has 64 rows of one head of two values."""
    rows = (1 << 28) + 1000
    x = torch.randn(1 << 20, 2, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda().repeat((rows >> 20) + 1, 1)[:rows].contiguous()
    positions = torch.arange(rows, dtype=torch.int32, device="cuda") % 1003
    turns = torch.tensor([0.01], dtype=torch.float64, device="cuda")
    y = torch.full_like(x, float("nan"))
    dnb.dnb_op_qk_rope_forward(dnb.dnb_qk_layout(rows, 1, 0, 2, 2), x, None, None, None, positions, turns, y, None)
    for a in range(0, rows, 1 << 24):
        part = x[a:a + (1 << 24)].float()
        angle = positions[a:a + (1 << 24)].double() * 0.01 * 2 * math.pi
        c, s = torch.cos(angle).float(), torch.sin(angle).float()
        want = torch.stack((part[:, 0] * c - part[:, 1] * s, part[:, 1] * c + part[:, 0] * s), 1)
        # half a step of bf16 of the result, and some 40 of fp32 of the terms on either side
        tol = want.abs() * 2.0 ** -8 + part.abs().sum(1, keepdim=True) * 80 * 2.0 ** -24
        assert bool(((y[a:a + (1 << 24)].float() - want).abs() <= tol).all()), a


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,most", [(256, 1.1e18), (8, 6e18)])
def test_norms_up_to_the_range_of_their_sums(dnb, dtype, dim, most):
    """A head of equal magnitudes comes out as the weight with its signs; one whose sum of squares is infinite as 0."""
    dt = DTYPES[dtype]
    gen = torch.Generator().manual_seed(3)
    sign = torch.randint(0, 2, (40, 3, dim), generator=gen) * 2 - 1
    w = (torch.rand(dim, generator=gen) + 0.5)
    for size, factor in ((most, 1.0), (3e19, 0.0)):
        x = (sign * size).to(dt).cuda()
        y = torch.full_like(x, 9.0)
        code = dnb.DNB_BF16 if dtype == "bf16" else dnb.DNB_F32
        dnb.dnb_op_qk_rope_forward(dnb.dnb_qk_layout(40, 3, 0, dim, 0, dtype=code), x, None, w.cuda(), None, None, None, y, None)
        want = (sign * w * factor).double()
        # the sum of 256 squares and the root, the type's rounding (all of a head are rounded alike)
        tol = want.abs() * (torch.finfo(dt).eps / 2 + 300 * 2.0 ** -24)
        assert bool(((y.cpu().double() - want).abs() <= tol).all()), size
