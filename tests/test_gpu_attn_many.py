"""Attention over more sequences than a wave looks through without an index, in each form, and how its time grows."""
import numpy as np
import pytest
import torch

import attn_forms
from seq_util import assert_within
from test_gpu_attn import Problem, ints

pytestmark = pytest.mark.gpu


def lengths(n, seed, most_q, most_k, none=0.2):
    """Random lengths, a part of them zero, with long ones at the ends of a chunk of 64 sequences."""
    r = np.random.default_rng(seed)
    q, k = r.integers(0, most_q + 1, n), r.integers(0, most_k + 1, n)
    q[r.random(n) < none] = 0
    k[r.random(n) < none] = 0
    for i in (0, 63, 64, 127, min(128, n - 1), n - 1):
        q[i], k[i] = most_q, most_k
    return [int(x) for x in q], [int(x) for x in k]


# sequences: around the numbers from which on there is an index (split 128, tiles backward 192, forward 384), a chunk more
# or less, more than one round of the search (64 chunks)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("n", [128, 193, 384, 385, 449, 4200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles(dnb, dtype, n, causal):
    q, k = lengths(n, n, 40 if n < 1000 else 3, 50 if n < 1000 else 5)
    p = Problem(dnb, dtype, q, k, 4, 2, 32, causal)
    attn_forms.check(dnb, p, "four")
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("n", [128, 129, 193, 4200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_split(dnb, dtype, n):
    """Single tokens and a few drafted ones over caches whose unused room holds NaN."""
    q, k = lengths(n, n + 1, 3, 400 if n < 1000 else 12)
    room = [x + 220 if n < 1000 else 205 for x in k]
    p = Problem(dnb, dtype, q, k, 4, 2, 32, True, capacity=room)
    attn_forms.check(dnb, p, "split")
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("split", [True, False])
def test_offsets_outside_the_tensors_are_cut_and_decreasing_ones_stay_inside(dnb, split):
    n = 400
    q, k = lengths(n, 5, 3, 400 if split else 30, none=0.0)
    p = Problem(dnb, "bf16", q, k, 4, 2, 32, True, capacity=[x + 200 for x in k] if split else None)
    attn_forms.check(dnb, p, "split" if split else "four")
    out, lse = p.forward()
    grads = p.backward(out, lse)
    big, good = 2 ** 31 - 1, p.o_
    p.o_ = (torch.cat([ints([-5]), good[0][1:-1], ints([big])]), torch.cat([ints([-big]), good[1][1:-1], ints([big])]), good[2])
    o, l = p.forward()
    assert torch.equal(o, out) and torch.equal(l, lse) and all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    r = np.random.default_rng(1)
    p.o_ = tuple(ints(r.integers(-9, 2 * t.shape[0], n + 1)) for t in (p.q, p.k)) + (ints(r.integers(-9, 500, n)),)
    p.backward(*p.forward())   # what comes out is undefined
    p.close()


@pytest.mark.parametrize("split", [True, False])
def test_rows_before_and_after_all_sequences_are_not_written(dnb, split):
    n = 400
    q, k = lengths(n, 6, 3, 400 if split else 30, none=0.1)
    q[0], q[-1] = q[0] + 5, q[-1] + 4
    p = Problem(dnb, "bf16", q, k, 4, 2, 32, True, capacity=[x + 200 for x in k] if split else None)
    attn_forms.check(dnb, p, "split" if split else "four")
    first, last = 5, sum(q) - 4
    p.qo[0], p.qo[-1] = first, last
    p.o_ = (ints(p.qo), *p.o_[1:])
    out, lse = p.forward()
    o, l, to, tl = p.oracle()
    mine = slice(first, last)
    assert_within(out[mine], o[mine], to[mine], "out")
    assert_within(lse[:, mine], l[:, mine], tl[:, mine], "lse")
    dq = p.backward(out, lse)[0]
    for t in (out, lse.T, dq):
        assert bool(torch.isnan(t[:first].float()).all()) and bool(torch.isnan(t[last:].float()).all())
        assert not bool(torch.isnan(t[mine].float()).any())
    p.close()


def test_repeats_bit_for_bit_in_a_graph(dnb):
    q, k = lengths(200, 9, 3, 600)
    p = Problem(dnb, "bf16", q, k, 4, 2, 64, True)
    attn_forms.check(dnb, p, "split")
    out, lse = torch.empty_like(p.dq_), torch.empty((4, p.q.shape[0]), device="cuda")
    dq, dk, dv, dout = torch.empty_like(p.dq_), torch.empty_like(p.dk_), torch.empty_like(p.dv_), p.dout.cuda()

    def calls():
        dnb.dnb_attn_forward(p.plan, p.dq_, p.dk_, p.dv_, *p.o_, out, lse, p.ws)
        dnb.dnb_attn_backward(p.plan, p.dq_, p.dk_, p.dv_, out, lse, dout, *p.o_, dq, dk, dv, p.ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        p.dq_.copy_(torch.randn(p.q.shape, generator=torch.Generator().manual_seed(turn)).to(p.dt))
        p.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, dq, dk, dv)]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, dq, dk, dv)))
    p.close()


def test_time_grows_with_the_number_of_sequences_and_not_its_square(dnb):
    """Four times the requests take no more than eight times as long (thirteen times with a walk through all of them)."""
    def times(n):
        q, k = torch.randn(n, 32, 64, device="cuda").bfloat16(), torch.randn(n * 256, 2, 64, device="cuda").bfloat16()
        v, out, lse = torch.randn_like(k), torch.empty_like(q), torch.empty(32, n, device="cuda")
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        qo = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        plan = dnb.dnb_attn_create(32, 2, 64, n, n, n * 256, causal=True)
        ws = torch.empty(dnb.dnb_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        got = []
        for call in (lambda: dnb.dnb_attn_forward(plan, q, k, v, qo, qo * 256, None, out, lse, ws),
                     lambda: dnb.dnb_attn_backward(plan, q, k, v, out, lse, q, qo, qo * 256, None, dq, dk, dv, ws)):
            best = float("inf")
            for _ in range(4):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                call()
                b.record()
                torch.cuda.synchronize()
                best = min(best, a.elapsed_time(b))
            got.append(best)
        dnb.dnb_attn_destroy(plan)
        return got

    few, many = times(1024), times(4096)
    print(few, many)
    assert many[0] <= 8 * few[0] and many[1] <= 8 * few[1], (few, many)


def test_no_workspace_is_refused(dnb):
    """The index lies in the workspace: without queries too."""
    plan = dnb.dnb_attn_create(4, 2, 32, 200, 0, 1000)
    k, off = torch.zeros(1000, 2, 32, dtype=torch.bfloat16, device="cuda"), ints([0] * 201)
    with pytest.raises(dnb.DnbError) as e:
        dnb.dnb_attn_backward(plan, None, k, k, None, None, None, off, off, None, None, torch.empty_like(k), torch.empty_like(k), None)
    assert e.value.status == dnb.DNB_E_NULL
    dnb.dnb_attn_destroy(plan)


@pytest.mark.parametrize("dim", [8, 64, 96, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_size_of_head(dnb, dtype, dim):
    """Key items of 64 and of 128 keys, in both types, and the split form's registers at every block count."""
    q, k = lengths(390, dim, 30, 40)
    p = Problem(dnb, dtype, q, k, 2, 1, dim, True)
    attn_forms.check(dnb, p, "four")
    p.check_forward()
    p.check_backward()
    p.close()
    q, k = lengths(140, dim, 3, 350, none=0.05)
    p = Problem(dnb, dtype, q, k, 4, 2, dim, True, capacity=[x + 130 for x in k])
    attn_forms.check(dnb, p, "split")
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_eight_waves(dnb, dtype):
    """Enough sequences for an index in the backward pass, and few enough tiles for eight waves."""
    r = np.random.default_rng(4)
    q, k = [int(x) for x in r.integers(0, 68, 195)], [int(x) for x in r.integers(0, 540, 195)]
    p = Problem(dnb, dtype, q, k, 1, 1, 32, True)
    attn_forms.check(dnb, p, "eight")
    p.check_forward()
    p.check_backward()
    p.close()
