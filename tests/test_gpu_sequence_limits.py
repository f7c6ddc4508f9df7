"""Sequence operators at the sizes where a launch has 2^24 workgroups and more, and where key positions reach 2^31."""
import math

import pytest
import torch

import attn_forms
from seq_util import assert_within, attn_backward, attn_forward, half_step
from test_gpu_attn import ints

pytestmark = pytest.mark.gpu


def room(gb):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gb * 2 ** 30:
        pytest.skip(f"needs {gb} GiB of device memory")


def test_rotary_rows_beyond_2_24_workgroups(dnb):
    """Rows of 1024 pairs, a workgroup each: in place, since they take 64 GiB."""
    rows, heads, dim = (1 << 24) + 3, 1024, 2
    room(75)
    x = torch.full((rows, heads, dim), 1.0, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    turns = torch.tensor([0.37 / (2 * math.pi)], dtype=torch.float64, device="cuda")
    dnb.dnb_op_rope_forward(x, pos, turns, x, rows, heads, dim, dim, dnb.DNB_ROPE_HALF, 1.0, dnb.DNB_BF16)
    angle = pos.double() * 0.37
    want = torch.stack((torch.cos(angle) - torch.sin(angle), torch.cos(angle) + torch.sin(angle)), 1)
    # as in test_gpu_rope.py: 8 steps of 2^-24 of |a| + |b| = 2, one rounding, and the product's in 64 bits
    tol = half_step(torch.bfloat16) * want.abs() + 16 * 2.0 ** -24 + 2 * rows * 2.0 ** -52
    assert bool(((x[:, 0].double() - want).abs() <= tol).all())
    for a in range(0, rows, 1 << 19):
        part = x[a:a + (1 << 19)]
        assert bool((part == part[:, :1]).all()), a
    del x, part


def test_split_form_with_2_24_rows_of_heads(dnb):
    """A workgroup joins a (row, head) of the split form: forward and dq, of requests of which few have keys."""
    n, heads, kv, dim = 4097, 4096, 128, 8
    rk = 200 * (n + 1)
    lengths = [40 if i % 997 == 0 else 300 if i == n - 1 else 0 for i in range(n)]
    assert attn_forms.form("bf16", [1] * n, rk, heads, kv) == "split" and n * heads >= 1 << 24
    room(20)
    gen = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16)
    mine = [i for i, x in enumerate(lengths) if x]
    q_few, do_few = rand(len(mine), heads, dim), rand(len(mine), heads, dim)
    k_few, v_few = rand(sum(lengths), kv, dim), rand(sum(lengths), kv, dim)
    q, dout = (torch.ones((n, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q[mine], dout[mine] = q_few.cuda(), do_few.cuda()
    k, v = (torch.empty((rk, kv, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:sum(lengths)], v[:sum(lengths)] = k_few.cuda(), v_few.cuda()
    ko = [0]
    for x in lengths:
        ko.append(ko[-1] + x)
    qo, ko_ = torch.arange(n + 1, dtype=torch.int32, device="cuda"), ints(ko)
    plan = dnb.dnb_attn_create(heads, kv, dim, n, n, rk, causal=True)
    ws = torch.empty(dnb.dnb_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full((heads, n), float("nan"), device="cuda")
    dnb.dnb_attn_forward(plan, q, k, v, qo, ko_, None, out, lse, ws)
    torch.cuda.synchronize()
    few_o = list(range(len(mine) + 1))
    few_k = [0] + [ko[i + 1] for i in mine]
    # heads of some groups only, so that the definition stays small
    pick = [0, 1, 31, 32, 2048, 4064, 4095]
    groups = sorted({h // (heads // kv) for h in pick})
    none = [i for i, x in enumerate(lengths) if not x]
    assert bool((out[none] == 0).all()) and bool((lse[:, none] == -math.inf).all())
    assert not bool(torch.isnan(out.float()).any()) and not bool(torch.isnan(lse).any())
    for h in pick:
        g = h // (heads // kv)
        o, l, to, tl = attn_forward(q_few[:, h:h + 1], k_few[:, g:g + 1], v_few[:, g:g + 1], few_o, few_k, None, True)
        assert_within(out[mine, h:h + 1], o, to, f"out of head {h}")
        assert_within(lse[h:h + 1, mine], l, tl, f"lse of head {h}")
    dq, dk, dv = torch.full_like(q, float("nan")), torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    dnb.dnb_attn_backward(plan, q, k, v, out, lse, dout, qo, ko_, None, dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert bool((dq[none] == 0).all()) and not bool(torch.isnan(dq.float()).any())
    used = sum(lengths)
    for g in groups:
        hs = slice(g * (heads // kv), (g + 1) * (heads // kv))
        o, l = out[mine][:, hs].cpu(), lse[hs][:, mine].cpu()
        want, tol = attn_backward(q_few[:, hs], k_few[:, g:g + 1], v_few[:, g:g + 1], o, l, do_few[:, hs], few_o, few_k, None, True)
        for got, w, t, name in zip((dq[mine][:, hs], dk[:used, g:g + 1], dv[:used, g:g + 1]), want, tol, ("dq", "dk", "dv")):
            assert_within(got, w, t, f"{name} of group {g}")
    assert bool(torch.isnan(dk[used:].float()).all()) and bool(torch.isnan(dv[used:].float()).all())   # rows of no sequence
    dnb.dnb_attn_destroy(plan)


def test_key_positions_up_to_2_31(dnb):
    """One query over 2^31 - 1 keys, all zero but the last two: one takes the weight, one is as the others."""
    nk, dim = 2 ** 31 - 1, 8
    room(165)
    k, v, dk, dv = (torch.zeros((nk, 1, dim), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    q = torch.full((1, 1, dim), 2.0, dtype=torch.bfloat16, device="cuda")
    k[-2] = 8.0                                  # score 2 * 8 * 8 / sqrt(8) = 45.25
    v[-2] = torch.arange(dim).to(torch.bfloat16).cuda()
    v[-1] = 2.0 ** 60                            # weight 2.2e-20: adds 0.0255 to every value
    score = 128 / math.sqrt(8)
    plan = dnb.dnb_attn_create(1, 1, dim, 1, 1, nk, causal=True)
    ws = torch.empty(dnb.dnb_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full((1, 1), float("nan"), device="cuda")
    off, ends = ints([0, 1]), ints([0, nk])
    dnb.dnb_attn_forward(plan, q, k, v, off, ends, None, out, lse, ws)
    torch.cuda.synchronize()
    r, f = half_step(torch.bfloat16), 2.0 ** -24
    want_lse = score + math.log1p((nk - 1) * math.exp(-score))
    # the score's products are exact, the scaled score is rounded some times: e, which a weight takes over
    e = f * (8 * score + 16)
    assert abs(float(lse) - want_lse) <= e
    small = math.exp(-want_lse)
    want = torch.arange(dim, dtype=torch.float64) * math.exp(score - want_lse) + small * 2.0 ** 60
    assert_within(out[0, 0], want, (2 * r + 2 * e) * want, "out")
    dout = torch.ones_like(q)
    dnb.dnb_attn_backward(plan, q, k, v, out, lse, dout, off, ends, None, q.clone(), dk, dv, ws)
    torch.cuda.synchronize()
    # dv: the weight of each key, once rounded to bf16 for its product and once at the end
    assert bool((dv[:-2] == dv[0]).all()) and bool((dv[-1] == dv[0]).all())
    assert abs(float(dv[0, 0, 0]) - small) <= (2 * r + 2 * e) * small and abs(float(dv[-2, 0, 0]) - 1) <= 2 * r + 2 * e
    # dk of a key of value 0: weight times (0 - sum dout out) times the query, over sqrt(8); sum dout out as out gives it
    D = float(out.double().sum())
    one = -small * D * 2 / math.sqrt(8)
    assert bool((dk[:-2] == dk[0]).all())
    assert abs(float(dk[0, 0, 0]) - one) <= (2 * r + 2 * e + 16 * f) * abs(one)
    last = small * (8 * 2.0 ** 60 - D) * 2 / math.sqrt(8)
    assert abs(float(dk[-1, 0, 0]) - last) <= (2 * r + 2 * e + 32 * f) * abs(last)
    dnb.dnb_attn_destroy(plan)
