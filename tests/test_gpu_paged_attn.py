"""Attention of new tokens over a paged cache against softmax(scale q k^T) v in 64 bits; the bounds on what rounding may add are
seq_util's."""
import math

import numpy as np
import pytest
import torch

from paged_util import LAYOUTS, Cache, ints, offsets
from seq_util import DTYPES, assert_within, attn_forward

pytestmark = pytest.mark.gpu


def run(dnb, cache, q, new, heads, causal=True, scale=0.0, out=None, lse=None, stream=None, q_offsets=None, lengths=None, table=None):
    n = q.shape[0]
    plan = dnb.dnb_paged_attn_create(cache.layout_of(dnb), heads, n, causal=causal, scale=scale, q_stride=q.stride(0) if n else 0)
    ws = torch.full((dnb.dnb_paged_attn_workspace_bytes(plan),), 0xff, dtype=torch.uint8, device="cuda")
    k, v = cache.to_gpu()
    if out is None:
        out = torch.full((n, heads, cache.dim), 7.0, dtype=cache.dtype, device="cuda")
    if lse is None:
        lse = torch.full((heads, n), 7.0, device="cuda")
    dnb.dnb_paged_attn_forward(plan, q, k, v, ints(offsets(new)) if q_offsets is None else q_offsets, ints(cache.lengths) if lengths is None else lengths,
                               ints(cache.table) if table is None else table, out, lse, ws, stream=stream)
    torch.cuda.synchronize()
    dnb.dnb_paged_attn_destroy(plan)
    return out, lse


def check(dnb, cache, new, heads, causal=True, scale=0.0, seed=1):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(sum(new), heads, cache.dim, generator=gen).to(cache.dtype)
    out, lse = run(dnb, cache, q.cuda(), new, heads, causal, scale)
    want, lwant, tol, ltol = attn_forward(q, cache.k, cache.v, offsets(new), cache.k_offsets, None, causal, scale or None)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("page", [1, 8, 16, 64, 256])
def test_pages_and_layouts(dnb, dtype, layout, page):
    cache = Cache([100, 1, 0, 63, 257], page, 2, 64, DTYPES[dtype], layout, columns=1 + 257 // page)
    check(dnb, cache, [1, 1, 0, 63, 30], 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_head_dims(dnb, dtype, dim):
    check(dnb, Cache([77, 150], 16, 2, dim, DTYPES[dtype]), [77, 3], 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (7, 1), (12, 4), (32, 1), (40, 1), (24, 8)])
def test_groups_of_heads(dnb, dtype, heads, kv):
    check(dnb, Cache([45, 333, 9], 16, kv, 32, DTYPES[dtype]), [45, 1, 2], heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 31), (1, 32), (1, 33), (1, 64), (1, 129), (2, 64), (16, 64), (17, 65), (31, 1000), (33, 500), (64, 64),
                                   (65, 127), (127, 128), (128, 129), (129, 300), (5, 3), (300, 7), (70, 0), (1, 0)])
def test_queries_and_keys(dnb, dtype, causal, nq, nk):
    """Among them more queries than keys, whose first see nothing, and no keys at all."""
    check(dnb, Cache([nk], 16, 2, 64, DTYPES[dtype]), [nq], 4, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_keys_are_shared_by_workgroups(dnb, dtype):
    check(dnb, Cache([20000], 16, 1, 64, DTYPES[dtype]), [1], 4)
    check(dnb, Cache([9000, 3, 5000], 32, 2, 128, DTYPES[dtype]), [40, 1, 1], 6)
    check(dnb, Cache([4100], 16, 1, 32, DTYPES[dtype]), [300], 2, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [65, 256, 257, 700])
def test_many_sequences(dnb, dtype, n):
    rng = np.random.default_rng(n)
    lengths = rng.integers(0, 60, n)
    new = np.minimum(rng.integers(0, 3, n), np.maximum(lengths, 0) + (rng.random(n) < 0.1))
    check(dnb, Cache(lengths.tolist(), 16, 2, 32, DTYPES[dtype]), new.tolist(), 4)


def test_a_batch_of_empty_places(dnb):
    cache = Cache([0, 0, 50, 0], 16, 2, 32, torch.bfloat16)
    check(dnb, cache, [0, 0, 2, 0], 4)
    check(dnb, cache, [0, 0, 0, 0], 4)


def test_many_places_without_requests(dnb):
    lengths = [0] * 1000 + [70] + [0] * 500 + [33]
    new = [0] * 1000 + [2] + [0] * 500 + [1]
    check(dnb, Cache(lengths, 16, 1, 32, torch.bfloat16), new, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scale_and_large_scores(dnb, dtype):
    check(dnb, Cache([300], 16, 2, 64, DTYPES[dtype], scale=4.0), [50], 4, scale=0.7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_in_the_rows_of_one_product(dnb, dtype):
    """q has a row stride; rows behind the last sequence's are left as they are, and lse may be null."""
    cache = Cache([90, 20], 16, 2, 64, DTYPES[dtype])
    gen = torch.Generator().manual_seed(3)
    rows = torch.randn(30, (4 + 2 * 2) * 64, generator=gen).to(DTYPES[dtype]).cuda()
    q, new = rows[:, :256], [20, 5]
    out, lse = run(dnb, cache, q, new, 4)
    want, lwant, tol, ltol = attn_forward(q[:25].reshape(25, 4, 64).cpu(), cache.k, cache.v, offsets(new), cache.k_offsets, None, True)
    assert_within(out[:25], want, tol, "out")
    assert_within(lse[:, :25], lwant, ltol, "lse")
    assert (out[25:] == 7).all() and (lse[:, 25:] == 7).all()
    plan = dnb.dnb_paged_attn_create(cache.layout_of(dnb), 4, 30, q_stride=rows.shape[1])
    ws = torch.empty(dnb.dnb_paged_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    again = torch.zeros_like(out)
    dnb.dnb_paged_attn_forward(plan, q, *cache.to_gpu(), ints(offsets(new)), ints(cache.lengths), ints(cache.table), again, None, ws)
    assert torch.equal(again[:25], out[:25])
    dnb.dnb_paged_attn_destroy(plan)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_not_of_the_pool(dnb, dtype):
    """Their keys and values are zeros."""
    cache = Cache([100], 16, 2, 64, DTYPES[dtype])
    q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype])
    table = cache.table.copy()
    table[0, 2], table[0, 4], table[0, 5] = -1, cache.pages, -2 ** 31
    out, lse = run(dnb, cache, q.cuda(), [3], 4, table=ints(table))
    k, v = cache.k.clone(), cache.v.clone()
    for a, b in ((32, 48), (64, 96)):
        k[a:b], v[a:b] = 0, 0
    want, lwant, tol, ltol = attn_forward(q, k, v, [0, 3], [0, 100], None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")


def test_lengths_and_offsets_that_leave_the_tensors(dnb):
    """Cut to the table's width and to the rows; negative lengths are none."""
    cache = Cache([64, 64, 5], 16, 1, 32, torch.bfloat16)
    q = torch.randn(6, 2, 32, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    out, lse = run(dnb, cache, q.cuda(), None, 2, q_offsets=ints([-3, 2, 4, 900]), lengths=ints([2 ** 31 - 1, -5, 5]))
    want, lwant, tol, ltol = attn_forward(q, torch.cat([cache.k[:64], cache.k[128:]]), torch.cat([cache.v[:64], cache.v[128:]]), [0, 2, 4, 6],
                                          [0, 64, 64, 69], None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")


def test_infinities_in_fp32(dnb):
    """What is seen and infinite is what arithmetic makes of it; what is hidden does nothing."""
    cache = Cache([80], 16, 1, 32, torch.float32)
    k, v = cache.k.clone(), cache.v.clone()
    v[70, 0, 3], v[75, 0, 4], v[20, 0, 5] = math.inf, math.nan, -math.inf
    k[79, 0, :] = 3.4e38
    for j in range(80):
        p, r = cache.table[0, j // 16], j % 16
        cache.k_pool[p, r], cache.v_pool[p, r] = k[j], v[j]
    q = torch.full((20, 2, 32), 1e-3)
    out, lse = run(dnb, cache, q.cuda(), [20], 2)
    out = out.cpu()
    last = torch.arange(20) + 60   # the last key that each query sees
    assert (out[:, :, 5] == -math.inf)[:19].all()
    assert ((out[:, :, 3] == math.inf) == (last >= 70)[:, None])[:19].all()
    assert (torch.isnan(out[:, :, 4]) == (last >= 75)[:, None])[:19].all()
    assert torch.isfinite(out[:19][:, :, [0, 1, 2, 6, 7]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeats_bit_for_bit_and_in_a_graph(dnb, dtype):
    """One captured graph follows lengths, offsets and table as they change, and two graphs share a workspace in turn."""
    cache = Cache([3000, 500, 64], 16, 2, 64, DTYPES[dtype])
    heads, q = 8, torch.randn(40, 8, 64, generator=torch.Generator().manual_seed(7)).to(DTYPES[dtype]).cuda()
    k, v = cache.to_gpu()
    plan = dnb.dnb_paged_attn_create(cache.layout_of(dnb), heads, 40)
    ws = torch.empty(dnb.dnb_paged_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    qo, kl, table = ints([0, 1, 30, 40]), ints(cache.lengths), ints(cache.table)
    outs = [torch.zeros(40, heads, 64, dtype=DTYPES[dtype], device="cuda") for _ in range(3)]
    lses = [torch.zeros(heads, 40, device="cuda") for _ in range(3)]

    def call(i):
        dnb.dnb_paged_attn_forward(plan, q, k, v, qo, kl, table, outs[i], lses[i], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        call(0)
        torch.cuda.synchronize()
        for i in (1, 2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(i)
            graphs.append(g)
    for offs, lengths in (([0, 1, 30, 40], [3000, 500, 64]), ([0, 20, 20, 30], [2777, 1, 60]), ([0, 0, 1, 2], [0, 500, 33])):
        qo.copy_(ints(offs))
        kl.copy_(ints(lengths))
        for i in range(3):
            outs[i].fill_(9)
            lses[i].fill_(9)
        call(0)
        for g in graphs * 2:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        assert torch.equal(lses[0], lses[1]) and torch.equal(lses[0], lses[2])
        ks = torch.cat([cache.k[o:o + n] for o, n in zip(cache.k_offsets, lengths)])
        vs = torch.cat([cache.v[o:o + n] for o, n in zip(cache.k_offsets, lengths)])
        n = offs[-1]
        want, lwant, tol, ltol = attn_forward(q[:n].cpu(), ks, vs, offs, offsets(lengths), None, True)
        assert_within(outs[0][:n], want, tol, "out")
        assert (outs[0][n:] == 9).all()
    dnb.dnb_paged_attn_destroy(plan)


def test_a_pool_past_32_bits(dnb):
    """Pages whose rows lie more than 2^31 elements into the pool."""
    page, kv, dim = 16, 8, 128
    pages = 2 ** 32 // (page * kv * dim) // 2 * 2 + 40   # 2^32 elements and some
    pool = torch.empty(pages, page, kv, dim, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(8)
    table = np.array([[pages - 1, 3, pages - 20, pages // 2 + 1]], dtype=np.int32)
    k, v = (torch.randn(60, kv, dim, generator=gen).to(torch.bfloat16) for _ in range(2))
    both = []
    for t in (k, v):
        p = pool if not both else torch.empty_like(pool)
        for j in range(60):
            p[int(table[0, j // page]), j % page] = t[j].cuda()
        both.append(p)
    q = torch.randn(2, 16, dim, generator=gen).to(torch.bfloat16)
    layout = dnb.dnb_paged_layout(pages, page, kv, dim, 1, 4)
    plan = dnb.dnb_paged_attn_create(layout, 16, 2)
    ws = torch.empty(dnb.dnb_paged_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(2, 16, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(16, 2, device="cuda")
    dnb.dnb_paged_attn_forward(plan, q.cuda(), *both, ints([0, 2]), ints([60]), ints(table), out, lse, ws)
    want, lwant, tol, ltol = attn_forward(q, k, v, [0, 2], [0, 60], None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")
    dnb.dnb_paged_attn_destroy(plan)
