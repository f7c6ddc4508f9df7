"""Attention over pages where scores and values span wide ranges: scores that leave a block of rows' first ones far behind, first
keys that weigh nothing, infinities, and shapes whose rows or keys straddle the kernels' steps."""
import math

import pytest
import torch

from paged_util import Cache, ints, offsets
from seq_util import DTYPES, assert_within, attn_forward
from test_gpu_paged_attn import check, run

pytestmark = pytest.mark.gpu

SHAPES = [([1], [700]), ([1, 1], [9000, 40]), ([7], [300]), ([100], [600]), ([300, 1], [900, 500])]


def with_keys(cache, change):
    """The cache after change(sequence's keys, sequence's values), which are views."""
    for s, n in enumerate(cache.lengths):
        a = int(cache.k_offsets[s])
        change(cache.k[a:a + n], cache.v[a:a + n])
        for j in range(n):
            p, r = int(cache.table[s, j // cache.page]), j % cache.page
            cache.k_pool[p, r], cache.v_pool[p, r] = cache.k[a + j], cache.v[a + j]
    return cache


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["rise", "fall", "peak"])
@pytest.mark.parametrize("range_", [40, 60, 100, 2000])
@pytest.mark.parametrize("new,lengths", SHAPES)
def test_scores_that_leave_the_first_ones(dnb, dtype, form, range_, new, lengths):
    """By e^range_ in a sequence: within what the weights of one maximum may grow by, past it, and past fp32."""
    def change(k, v):
        at = torch.linspace(0, 1, len(k))
        if form == "fall":
            at = 1 - at
        if form == "peak":
            at = torch.zeros(len(k))
            at[int(len(k) * 0.77)] = 1
        k[:, :, 0] = (range_ * at[:, None]).to(k.dtype)
    cache = with_keys(Cache(lengths, 16, 2, 64, DTYPES[dtype]), change)
    q = torch.randn(sum(new), 8, 64, generator=torch.Generator().manual_seed(3)).to(DTYPES[dtype])
    q[:, :, 0] = 8.0    # times 1 / sqrt(64): the first coordinate is the score
    out, lse = run(dnb, cache, q.cuda(), new, 8)
    want, lwant, tol, ltol = attn_forward(q, cache.k, cache.v, offsets(new), cache.k_offsets, None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("none", [1, 40, 200])
@pytest.mark.parametrize("new,lengths", SHAPES)
def test_first_keys_that_weigh_nothing(dnb, dtype, none, new, lengths):
    """Scores of minus infinity: the results are those of the other keys.  And of all other keys' scores far below zero."""
    for far in (0.0, -3000.0):
        def change(k, v):
            k[:, :, 0] = far
            k[:min(none, len(k) // 3), :, 0] = -math.inf
        cache = with_keys(Cache(lengths, 16, 2, 64, DTYPES[dtype]), change)
        q = torch.randn(sum(new), 8, 64, generator=torch.Generator().manual_seed(4)).to(DTYPES[dtype])
        q[:, :, 0] = 8.0
        out, lse = run(dnb, cache, q.cuda(), new, 8)
        left = [n - min(none, n // 3) for n in lengths]
        k, v = (torch.cat([t[int(o) + n - m:int(o) + n] for o, n, m in zip(cache.k_offsets, lengths, left)]) for t in (cache.k, cache.v))
        want, lwant, tol, ltol = attn_forward(q, k, v, offsets(new), offsets(left), None, True)
        assert_within(out, want, tol, "out")
        assert_within(lse, lwant, ltol, "lse")


@pytest.mark.parametrize("new,lengths", SHAPES)
def test_infinities_in_bf16(dnb, new, lengths):
    """What is seen and infinite is what arithmetic makes of it, in its column and its sequence; NaN in a key is NaN in all that see it."""
    def change(k, v):
        v[5, 0, 3], v[len(v) // 2, 0, 4], v[0, 1, 5] = math.inf, math.nan, -math.inf
    cache = with_keys(Cache(lengths, 16, 2, 64, torch.bfloat16), change)
    q = torch.randn(sum(new), 8, 64, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    out = run(dnb, cache, q.cuda(), new, 8)[0].cpu()
    last = torch.cat([torch.arange(n) + m - n for n, m in zip(new, lengths)])
    half = torch.cat([torch.full((n,), m // 2) for n, m in zip(new, lengths)])
    assert (out[last >= 5][:, :4, 3] == math.inf).all() and torch.isnan(out[last >= half][:, :4, 4]).all()
    assert (out[:, 4:, 5] == -math.inf).all()
    rest = [c for c in range(64) if c not in (3, 4, 5)]
    assert torch.isfinite(out[:, :, rest]).all() and torch.isfinite(out[:, 4:, 3:5]).all() and torch.isfinite(out[:, :4, 5]).all()

    def nan_key(k, v):
        v[:] = 1.0
        k[len(k) - 1, 1, 7] = math.nan
    cache = with_keys(Cache(lengths, 16, 2, 64, torch.bfloat16), nan_key)
    out = run(dnb, cache, q.cuda(), new, 8)[0].cpu()
    seen = last == torch.cat([torch.full((n,), m - 1) for n, m in zip(new, lengths)])
    assert torch.isnan(out[seen][:, 4:]).all() and torch.isfinite(out[:, :4]).all()
    assert torch.isfinite(out[~seen]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(50, 300), (63, 129), (64, 512), (65, 511), (120, 300), (128, 1025), (129, 640), (260, 700), (513, 513), (257, 130)])
@pytest.mark.parametrize("dim", [40, 128])
def test_rows_that_straddle_steps(dnb, dtype, nq, nk, dim):
    """One query head a key/value head and three: sets of rows that end within a wave's, within a block's, and a row past them."""
    for heads in (1, 3):
        check(dnb, Cache([nk], 32, 1, dim, DTYPES[dtype]), [nq], heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_and_tokens_in_one_batch(dnb, dtype):
    """Blocks of each kind side by side on the line, among them sequences without new tokens, without keys, and with more new tokens than keys."""
    new = [1, 0, 300, 1, 17, 40, 3, 1, 0, 90, 5]
    lengths = [2000, 77, 700, 1, 17, 1300, 0, 0, 5, 60, 4000]
    for causal in (True, False):
        check(dnb, Cache(lengths, 16, 2, 128, DTYPES[dtype]), new, 8, causal)


def test_on_another_stream_than_the_tensors(dnb):
    cache = Cache([500, 90], 16, 2, 64, torch.bfloat16)
    q = torch.randn(31, 4, 64, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    first, _ = run(dnb, cache, q, [1, 30], 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, _ = run(dnb, cache, q, [1, 30], 4, stream=side)
    assert torch.equal(first, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 20, 90, 400])
def test_pages_not_of_the_pool_in_long_sequences(dnb, dtype, nq):
    """Zeros, in steps among others whose pages are all there, and in the first and the last."""
    cache = Cache([2100], 16, 1, 128, DTYPES[dtype])
    q = torch.randn(nq, 4, 128, generator=torch.Generator().manual_seed(7)).to(DTYPES[dtype])
    table, k, v = cache.table.copy(), cache.k.clone(), cache.v.clone()
    for page, at in ((-1, 0), (cache.pages, 9), (2 ** 31 - 1, 40), (-2 ** 31, 41), (cache.pages + 7, 100), (-5, 131)):
        table[0, at] = page
        k[16 * at:16 * at + 16], v[16 * at:16 * at + 16] = 0, 0
    out, lse = run(dnb, cache, q.cuda(), [nq], 4, table=ints(table))
    want, lwant, tol, ltol = attn_forward(q, k, v, [0, nq], [0, 2100], None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [0, 2 ** 26])
@pytest.mark.parametrize("nq", [1, 150])
def test_rows_far_apart(dnb, dtype, gap, nq):
    """A pool of which the same row of all pages lies together, also with more than 2^26 elements from row to row."""
    page, kv, dim, keys = 4, 2, 32, 390
    pages = 100
    row = pages * kv * dim + gap
    pools = [torch.zeros((page - 1) * row + pages * kv * dim, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    gen = torch.Generator().manual_seed(8)
    k, v = (torch.randn(keys, kv, dim, generator=gen).to(DTYPES[dtype]) for _ in range(2))
    order = torch.randperm(pages, generator=gen)
    for t, pool in zip((k, v), pools):
        for r in range(page):
            rows = t[r::page]
            pool[r * row:r * row + pages * kv * dim].view(pages, kv, dim)[order[:len(rows)].cuda()] = rows.cuda()
    layout = dnb.dnb_paged_layout(pages, page, kv, dim, 1, 98, dtype=dnb.DNB_BF16 if dtype == "bf16" else dnb.DNB_F32, page_stride=kv * dim,
                                  row_stride=row, head_stride=dim)
    q = torch.randn(nq, 4, dim, generator=gen).to(DTYPES[dtype])
    plan = dnb.dnb_paged_attn_create(layout, 4, nq)
    ws = torch.empty(dnb.dnb_paged_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(nq, 4, dim, dtype=DTYPES[dtype], device="cuda"), torch.zeros(4, nq, device="cuda")
    dnb.dnb_paged_attn_forward(plan, q.cuda(), *pools, ints([0, nq]), ints([keys]), ints(order[:98].numpy()), out, lse, ws)
    torch.cuda.synchronize()
    dnb.dnb_paged_attn_destroy(plan)
    want, lwant, tol, ltol = attn_forward(q, k, v, [0, nq], [0, keys], None, True)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")
