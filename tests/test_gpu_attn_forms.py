"""Attention in each of its forms, by name: the form that splits the keys, tiles of four waves and of eight.
Every test says which form it runs and checks it (attn_forms.py)."""
import numpy as np
import pytest
import torch

import attn_forms
from seq_util import DTYPES, assert_within, attn_backward, attn_forward
from test_gpu_attn import Problem, ints

pytestmark = pytest.mark.gpu

DIMS = [32, 64, 96, 128]


def heads_for_tiles(rows, lo, hi):
    """Key/value heads, one query head each, with which (rows / 128 + 1) tiles a head make lo .. hi workgroups."""
    kv = -(-lo // (rows // 128 + 1))
    assert (-(-rows // 128) + 2) * kv <= hi
    return kv


# bf16 tiles: more than 40, fp32: more than 96; of eight waves: up to 256
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_eight_waves(dnb, dtype, dim, causal):
    """Long sequences with a remainder in rows and keys, more than one of the eight waves' double tiles."""
    per = 1 if dtype == "f32" else 2
    rows, n = (517, 1) if dtype == "f32" else (405, 1)
    kv = heads_for_tiles(rows * per, 97 if dtype == "f32" else 41, 250)
    p = Problem(dnb, dtype, [rows], [rows + 82], kv * per, kv, dim, causal)
    attn_forms.check(dnb, p, "eight")
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("dim", DIMS + [40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_eight_waves_with_a_short_sequence_and_more_queries_than_keys(dnb, dtype, dim):
    kv = 20 if dtype == "f32" else 9
    p = Problem(dnb, dtype, [430, 3, 150], [700, 70, 33], kv, kv, dim, True)
    attn_forms.check(dnb, p, "eight")
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("dtype,dim", [("bf16", 8), ("bf16", 32), ("f32", 8), ("f32", 32), ("bf16", 96), ("f32", 128)])
def test_split_keys_at_every_block_count(dnb, dtype, dim):
    p = Problem(dnb, dtype, [3, 50], [800, 500], 4, 2, dim, True)
    attn_forms.check(dnb, p, "split")
    p.check_forward()
    p.check_backward()
    p.close()


FORMS = {"split": ([1, 1, 1], [900, 800, 700], 4, 2), "four": ([100, 40, 7], [200, 64, 7], 4, 2), "eight": ([517], [599], 20, 20)}


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_a_graph(dnb, dtype, form):
    """Captured once and replayed on new values, with eager work between the replays."""
    q, k, heads, kv = FORMS[form]
    p = Problem(dnb, dtype, q, k, heads, kv, 64, True)
    attn_forms.check(dnb, p, form)
    out = torch.empty(p.q.shape, dtype=p.dt, device="cuda")
    lse = torch.empty((heads, p.q.shape[0]), device="cuda")
    dout = p.dout.cuda()
    dq, dk, dv = (torch.empty_like(t) for t in (p.dq_, p.dk_, p.dv_))

    def calls(stream):
        dnb.dnb_attn_forward(p.plan, p.dq_, p.dk_, p.dv_, *p.o_, out, lse, p.ws, stream=stream)
        dnb.dnb_attn_backward(p.plan, p.dq_, p.dk_, p.dv_, out, lse, dout, *p.o_, dq, dk, dv, p.ws, stream=stream)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(torch.cuda.current_stream())
    for turn in range(3):
        p.dq_.copy_(torch.randn(p.q.shape, generator=torch.Generator().manual_seed(turn)).to(p.dt))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, dq, dk, dv)]
        calls(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, dq, dk, dv)))
    p.close()


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeats_bit_for_bit(dnb, dtype, form):
    q, k, heads, kv = FORMS[form]
    p = Problem(dnb, dtype, q, k, heads, kv, 64, True)
    attn_forms.check(dnb, p, form)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    for _ in range(3):
        p.ws.fill_(255)
        o, l = p.forward()
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    p.close()


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
def test_offsets_outside_the_tensors_are_cut_to_them(dnb, form):
    q, k, heads, kv = FORMS[form]
    p = Problem(dnb, "bf16", q, k, heads, kv, 64, True)
    attn_forms.check(dnb, p, form)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    big = 2 ** 31 - 1
    p.o_ = (torch.cat([ints([-5]), p.o_[0][1:-1], ints([big])]), torch.cat([ints([-big]), p.o_[1][1:-1], ints([big])]), None)
    o, l = p.forward()
    assert torch.equal(o, out) and torch.equal(l, lse) and all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    # offsets that decrease: what comes out is undefined
    n = len(q)
    p.o_ = (ints([9, 2, big, -7][:n + 1]), ints([100, -3, 50, 7][:n + 1]), ints([big, 5, -1][:n]))
    p.backward(*p.forward())
    p.close()


@pytest.mark.parametrize("form", ["split", "four", "eight"])
def test_rows_past_32_bits(dnb, form):
    """Keys and queries whose elements lie beyond 2^31: rows 2^22 elements apart, forward and all gradients."""
    stride = 1 << 22
    q, k, kv = {"split": ([1, 3], [100, 500], 1), "four": ([400, 90, 100], [130, 90, 480], 9), "eight": ([40, 500], [60, 600], 9)}[form]
    dim, per = 32, 2 if form == "split" else 1
    p = Problem(dnb, "bf16", q, k, kv * per, kv, dim, True)
    attn_forms.check(dnb, p, form)
    rq, rk = sum(q), sum(k)
    # one matrix: queries, keys, values and their gradients side by side in its rows
    rows = max(rq, rk)
    assert (rk - 1) * stride > 2 ** 31
    buf = torch.empty(stride * rows, dtype=torch.bfloat16, device="cuda")
    view = lambda at, n, heads: buf[at * 1024:].as_strided((n, heads * dim), (stride, 1))
    qv, kk, vv = view(0, rq, kv * per), view(1, rk, kv), view(2, rk, kv)
    dq, dk, dv = view(3, rq, kv * per), view(4, rk, kv), view(5, rk, kv)
    qv.copy_(p.dq_.reshape(qv.shape))
    kk.copy_(p.dk_.reshape(kk.shape))
    vv.copy_(p.dv_.reshape(vv.shape))
    for t in (dq, dk, dv):
        t.fill_(float("nan"))
    dnb.dnb_attn_destroy(p.plan)
    p.plan = dnb.dnb_attn_create(kv * per, kv, dim, len(q), rq, rk, causal=True, q_stride=stride, k_stride=stride, v_stride=stride)
    p.ws = torch.full((dnb.dnb_attn_workspace_bytes(p.plan),), 255, dtype=torch.uint8, device="cuda")
    p.dq_, p.dk_, p.dv_ = qv, kk, vv
    p.check_forward()
    o, l, _, _ = p.oracle()
    out, lse = o.to(p.dt), l.float()
    dnb.dnb_attn_backward(p.plan, qv, kk, vv, out.cuda(), lse.cuda(), p.dout.cuda(), *p.o_, dq, dk, dv, p.ws)
    torch.cuda.synchronize()
    want, tol = attn_backward(p.q, p.k, p.v, out, lse, p.dout, p.qo, p.ko, None, True)
    for got, w, t, name in zip((dq, dk, dv), want, tol, ("dq", "dk", "dv")):
        assert_within(got.reshape(w.shape), w, t, name)
    p.close()
    del buf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_drafted_tokens_a_request_over_long_keys(dnb, dtype):
    """Several queries a request, over keys that are long enough to be split; unused room holds NaN."""
    p = Problem(dnb, dtype, [5, 1, 0, 40, 3, 2], [700, 1, 90, 900, 200, 0], 8, 4, 64, True, capacity=[800, 1, 120, 933, 202, 5])
    attn_forms.check(dnb, p, "split")
    p.check_forward()
    p.check_backward()
    p.close()


def test_gradients_of_rows_that_see_few_keys_are_as_exact_as_bf16_allows(dnb):
    """Rows that see up to 128 keys: ds in two parts and sum dout out from the weights, so that dq and dk have no
    rounding to bf16 but their own.  The weights are exp of scores and an lse in fp32: e of each below.

    What is left: dq = scale ds k has half a step of its own, and ds rounded twice: 2^-16 of its terms; an
    error e of every p changes ds by e (|ds| + p sum_j |ds_j|) at most."""
    lengths, heads, kv, dim = [33, 10, 1, 64, 100], 4, 2, 64
    p = Problem(dnb, "bf16", lengths, lengths, heads, kv, dim, True)
    o, l, _, _ = p.oracle()
    got = p.backward(o.to(p.dt).cuda(), l.float().cuda())
    r, f = 2.0 ** -8, 2.0 ** -24
    # the oracle with the definition's own out, not the rounded one
    (dq, dk, _), _ = attn_backward(p.q, p.k, p.v, o, l, p.dout, p.qo, p.ko, None, True)
    tq, tk = torch.zeros_like(dq), torch.zeros_like(dk)
    for a, b in zip(p.qo, p.qo[1:]):
        s = slice(a, b)
        hidden = torch.ones(b - a, b - a, dtype=torch.bool).triu(1)
        for h in range(heads):
            g = h // (heads // kv)
            q, k, v, do = (t.double() for t in (p.q[s, h], p.k[s, g], p.v[s, g], p.dout[s, h]))
            w = torch.softmax((q @ k.T / dim ** 0.5).masked_fill(hidden, -np.inf), 1)
            dp, size = do @ v.T, do.abs() @ v.abs().T
            D = (w * dp).sum(1, keepdim=True)
            ds = w * (dp - D)
            score = (q.abs() @ k.abs().T / dim ** 0.5).masked_fill(hidden, 0).amax(1, keepdim=True)
            e = f * ((dim + 8) * score + 4 * l[h, s][:, None].abs() + 16)
            # D sums b - a terms p dp in fp32, each e off; dp a sum of dim products
            es = e * ds.abs() + w * ((e + f * (b - a)) * (w * size).sum(1, keepdim=True) + f * (dim + 4) * (size + (w * size).sum(1, keepdim=True)))
            es = es + (2.0 ** -16 + f * (b - a) * (heads // kv)) * ds.abs()   # dk sums the rows of both heads
            tq[s, h] = es @ k.abs() / dim ** 0.5
            tk[s, g] += es.T @ q.abs() / dim ** 0.5
    assert_within(got[0], dq, tq + r * dq.abs(), "dq")
    assert_within(got[1], dk, tk + r * dk.abs(), "dk")
    p.close()
