"""Attention over pages where some rows' scores rise far above the first ones and other rows' do not, by amounts whose weights are still
finite in fp32: sums of several of them are not, nor are those of several waves and parts, and a part that began low must not be lost
beside one that began high.  The keys are so many that a workgroup's part has several steps; the rows that rise are not the first of any set of 32."""
import pytest
import torch

from paged_util import ints
from seq_util import DTYPES, assert_within, attn_forward

pytestmark = pytest.mark.gpu

KEYS, PAGE, DIM, STEP = 12000, 32, 32, 128
# queries, key/value heads, query heads of each, rows (query, then head) that rise: at most 32 rows, at most 128, more
SHAPES = {"narrow": (8, 8, 4, [1, 9, 31]), "half": (20, 8, 4, [33, 63, 70]), "wide": (150, 4, 2, [31, 33, 63, 255, 257])}


def peaks(form):
    """Keys with a high score, for rows that rise."""
    steps = range(2, KEYS // STEP - 2)
    if form == "lane":    # four that one lane of a wave adds up
        return [s * STEP + 40 + i for s in steps if s % 7 == 3 for i in range(4)]
    if form == "waves":   # one for each of four waves
        return [s * STEP + 32 * w + 6 for s in steps if s % 7 == 3 for w in range(4)]
    return [s * STEP + 75 for s in steps if s % 3 == 0]   # in some parts among the first keys, in others not


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["lane", "waves", "parts"])
@pytest.mark.parametrize("rise", [44.0, 60.0, 87.5])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_some_rows_rise(dnb, dtype, form, rise, shape):
    nq, kv, per, rows = SHAPES[shape]
    heads, dt, gen = kv * per, DTYPES[dtype], torch.Generator().manual_seed(int(rise))
    k, v = torch.randn(KEYS, kv, DIM, generator=gen), torch.randn(KEYS, kv, DIM, generator=gen) * 2.0 ** -6
    k[:, :, 0] = 0
    k[peaks(form), :, 0] = rise
    # the first coordinate is the score, but for some 0.1 of the others
    q = torch.randn(nq, heads, DIM, generator=gen) * 0.02
    q[:, :, 0] = 0
    for m in rows:
        q[m // per, m % per::per, 0] = 1
    q, k, v = (t.to(dt) for t in (q, k, v))
    pages = KEYS // PAGE
    order = torch.randperm(pages, generator=gen)
    pools = []
    for t in (k, v):
        pool = torch.empty(pages, PAGE, kv, DIM, dtype=dt)
        pool[order] = t.view(pages, PAGE, kv, DIM)
        pools.append(pool.cuda())
    layout = dnb.dnb_paged_layout(pages, PAGE, kv, DIM, 1, pages, dtype=dnb.DNB_BF16 if dtype == "bf16" else dnb.DNB_F32)
    plan = dnb.dnb_paged_attn_create(layout, heads, nq, scale=1.0)
    ws = torch.full((dnb.dnb_paged_attn_workspace_bytes(plan),), 0xff, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(nq, heads, DIM, dtype=dt, device="cuda"), torch.zeros(heads, nq, device="cuda")
    dnb.dnb_paged_attn_forward(plan, q.cuda(), *pools, ints([0, nq]), ints([KEYS]), ints(order.numpy()), out, lse, ws)
    torch.cuda.synchronize()
    dnb.dnb_paged_attn_destroy(plan)
    want, lwant, tol, ltol = attn_forward(q, k, v, [0, nq], [0, KEYS], None, True, 1.0)
    assert_within(out, want, tol, "out")
    assert_within(lse, lwant, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", [1e3, 1e6, 1e9, -1e9])
@pytest.mark.parametrize("nq", [1, 40, 150])
def test_scores_up_to_a_thousand_million(dnb, dtype, score, nq):
    """Two keys among many are far above all others, or all are equal: the weights are one half each, or all the same, whatever the scores'
    size, so that out is an average that rounding knows: of two values exact but for its own rounding and that of a weight 2^k, which
    divides out; of all, that of a sum of n."""
    keys, dt, gen = 2000, DTYPES[dtype], torch.Generator().manual_seed(5)
    k, v = torch.zeros(keys, 1, DIM), torch.randn(keys, 1, DIM, generator=gen).to(dt)
    k[:, :, 0] = -1
    far = [700, 1301]
    if score > 0:
        k[far, :, 0] = 1
    q = torch.zeros(nq, 2, DIM)
    q[:, :, 0] = abs(score)
    q, k = q.to(dt), k.to(dt)
    pages = -(-keys // PAGE)
    pools = [torch.nn.functional.pad(t, (0, 0, 0, 0, 0, pages * PAGE - keys)).view(pages, PAGE, 1, DIM).cuda() for t in (k, v)]
    layout = dnb.dnb_paged_layout(pages, PAGE, 1, DIM, 1, pages, dtype=dnb.DNB_BF16 if dtype == "bf16" else dnb.DNB_F32)
    plan = dnb.dnb_paged_attn_create(layout, 2, nq, scale=1.0)
    ws = torch.full((dnb.dnb_paged_attn_workspace_bytes(plan),), 0xff, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(nq, 2, DIM, dtype=dt, device="cuda"), torch.zeros(2, nq, device="cuda")
    dnb.dnb_paged_attn_forward(plan, q.cuda(), *pools, ints([0, nq]), ints([keys]), ints(range(pages)), out, lse, ws)
    torch.cuda.synchronize()
    dnb.dnb_paged_attn_destroy(plan)
    last = torch.arange(nq) + keys - nq + 1
    wide = v[:, 0].double()
    want = torch.stack([wide[far].mean(0) if score > 0 else wide[:n].mean(0) for n in last.tolist()])[:, None].expand(nq, 2, DIM)
    half = torch.finfo(dt).eps / 2
    # the weights are all the same number, whatever rounding has made of it; sums of n terms, one division, the type's rounding
    tol = half * want.abs() + 2.0 ** -24 * (keys + 4) * wide.abs().mean() * (1 if score < 0 else 4) + 2 * half * (wide.abs().mean() if score < 0 else wide[far].abs().mean())
    assert bool(((out.cpu().double() - want).abs() <= tol).all())
    assert bool((lse.cpu().double() - float(q[0, 0, 0]) * (1 if score > 0 else -1)).abs().max() <= 2.0 ** -20 * abs(score) + 8)
