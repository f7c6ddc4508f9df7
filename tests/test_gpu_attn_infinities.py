"""Infinities and the largest finite values in fp32 attention: what the definition gives, in the tiled form
and in the form that splits the keys alike."""
import math

import pytest
import torch

from seq_util import assert_within, attn_backward, attn_forward
from test_gpu_attn import Problem

pytestmark = pytest.mark.gpu

# (query lengths, key lengths, heads, kv_heads, head_dim): tiles of four waves, of eight, and the split form
FORMS = {"tile": ([70, 5], [70, 40], 4, 2, 64), "tile128": ([70, 5], [70, 40], 4, 2, 128), "eight": ([1300], [1300], 12, 12, 32),
         "eight128": ([1300], [1300], 12, 12, 128), "split": ([1, 2], [700, 900], 4, 2, 64)}


def same(got, want, tol, what):
    """Equal where the definition is infinite, NaN where it is, else within tol."""
    got = got.detach().double().cpu()
    assert bool((torch.isnan(got) == torch.isnan(want)).all()), what
    finite = torch.isfinite(want)
    keep = torch.isinf(want)
    assert bool((got[keep] == want[keep]).all()), what
    assert_within(got[finite], want[finite], tol[finite], what)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
def test_an_infinite_value_reaches_the_queries(dnb, form, sign):
    q, k, heads, kv, dim = FORMS[form]
    p = Problem(dnb, "f32", q, k, heads, kv, dim, False)
    p.v[3, 0, 5] = sign * math.inf
    p.v[k[0] - 1, kv - 1, dim - 1] = sign * math.inf
    p.dv_ = p.v.cuda()
    out, lse = p.forward()
    o, l, to, tl = p.oracle()
    assert bool(torch.isinf(o[:q[0]]).any()) and not bool(torch.isnan(o).any())
    same(out, o, torch.nan_to_num(to, posinf=0.0), "out")
    assert_within(lse, l, tl, "lse")
    p.close()


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
def test_an_infinite_key_takes_or_loses_all_weight(dnb, form):
    """A score of minus infinity has no weight; one of infinity leaves NaN, as inf - inf does."""
    q, k, heads, kv, dim = FORMS[form]
    p = Problem(dnb, "f32", q, k, heads, kv, dim, False)
    p.q = p.q.abs() + 0.5
    p.k[1:k[0] - 2] = -math.inf
    p.dq_, p.dk_ = p.q.cuda(), p.k.cuda()
    out, lse = p.forward()
    keep = [0] + list(range(k[0] - 2, sum(k)))
    o, l, to, tl = attn_forward(p.q, p.k[keep], p.v[keep], p.qo, [0] + [x - k[0] + 3 for x in p.ko[1:]], None, False)
    assert_within(out, o, to, "out")
    assert_within(lse, l, tl, "lse")
    p.k[1, 0, 0] = math.inf
    p.k[1, 0, 1:] = 0.0
    p.dk_ = p.k.cuda()
    out, _ = p.forward()
    assert bool(torch.isnan(out[:q[0], 0]).all())      # the query's own softmax is inf / inf
    same(out[q[0]:], o[q[0]:], to[q[0]:], "the other sequence")
    p.close()


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
def test_the_largest_finite_values(dnb, form):
    """Values between the largest bf16 and the largest fp32 are what they are: of keys with a score of 0, so that no
    sum before its division by the sum of the weights is larger than they."""
    q, k, heads, kv, dim = FORMS[form]
    p = Problem(dnb, "f32", q, k, heads, kv, dim, False)
    most = torch.finfo(torch.float32).max
    p.v[3, 0, 0], p.v[k[0] - 2, kv - 1, 1] = most, -0.9995 * most
    p.k[3], p.k[k[0] - 2] = 0.0, 0.0
    p.dv_, p.dk_ = p.v.cuda(), p.k.cuda()
    out, lse = p.forward()
    o, l, to, tl = p.oracle()
    assert_within(out, o, to, "out")
    assert_within(lse, l, tl, "lse")
    p.close()


@pytest.mark.parametrize("form", FORMS, ids=list(FORMS))
def test_infinite_gradients_stay_infinite(dnb, form):
    """One infinite value of dout: its sequence's dv and the dq, dk behind it are not finite, as by the definition; others are exact."""
    q, k, heads, kv, dim = FORMS[form]
    p = Problem(dnb, "f32", q, k, heads, kv, dim, False)
    o, l, _, _ = p.oracle()
    out, lse = o.float(), l.float()
    p.dout[0, heads - 1, 2] = math.inf
    dq, dk, dv = p.backward(out.cuda(), lse.cuda())
    want, tol = attn_backward(p.q, p.k, p.v, out, lse, p.dout, p.qo, p.ko, p.kl, False, 0.0)
    # dv: weight times infinity in one column of every key of the sequence and head
    same(dv, want[2], torch.nan_to_num(tol[2], posinf=0.0), "dv")
    assert bool(torch.isinf(dv[:k[0], kv - 1, 2]).all())
    # dq and dk: infinite minus infinite; which of the two a row gets depends on the order of its sum
    for g, w, t, name in ((dq, want[0], tol[0], "dq"), (dk, want[1], tol[1], "dk")):
        g = g.double().cpu()
        assert bool((torch.isfinite(g) == torch.isfinite(w)).all()), name
        f = torch.isfinite(w)
        assert_within(g[f], w[f], t[f], name)
    p.close()


MASKED = {"tile": ([70, 40], [70, 40], 4, 2, 64), "tile128": ([70, 40], [75, 40], 4, 2, 128), "eight": ([1300], [1300], 12, 12, 32),
          "eight128": ([1300], [1310], 12, 12, 128)}


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("form", MASKED, ids=list(MASKED))
def test_what_a_causal_mask_hides_does_not_matter(dnb, form, bad):
    """Keys, values, queries and dout from some row on: earlier queries do not see those keys, and later keys are not seen
    by those queries, whatever they hold.  Within one tile of 32, and in its tile's neighbours."""
    q, k, heads, kv, dim = MASKED[form]
    p = Problem(dnb, "f32", q, k, heads, kv, dim, True)
    shift, n = k[0] - q[0], 45
    good = [t.clone() for t in (p.q, p.k, p.v, p.dout)]
    o, l, to, tl = p.oracle()
    # forward and dq: a value, and a key, that queries from n on see
    for which in ("v", "k"):
        p.q, p.k, p.v, p.dout = (t.clone() for t in good)
        getattr(p, which)[n + shift, 0, 3] = bad
        p.dk_, p.dv_ = p.k.cuda(), p.v.cuda()
        out, lse = p.forward()
        same(out[:n], o[:n], to[:n], f"out, {which}")
        assert_within(lse[:, :n], l[:, :n], tl[:, :n], "lse")
        assert not bool(torch.isfinite(out[n:q[0], 0]).all())
        assert torch.equal(torch.isfinite(out[q[0]:]), torch.ones_like(out[q[0]:], dtype=torch.bool))
        out_, lse_ = o.float(), l.float()
        dq = p.backward(out_.cuda(), lse_.cuda())[0]
        (want, _, _), (tol, _, _) = attn_backward(good[0], good[1], good[2], out_, lse_, good[3], p.qo, p.ko, None, True)
        same(dq[:n], want[:n], tol[:n], f"dq, {which}")
    # dk and dv: a query, and a dout, that keys up to n + shift see
    want, tol = attn_backward(good[0], good[1], good[2], o.float(), l.float(), good[3], p.qo, p.ko, None, True)
    later = slice(n + shift + 1, k[0])
    for which in ("q", "dout"):
        p.q, p.k, p.v, p.dout = (t.clone() for t in good)
        getattr(p, which)[n, 0, 3] = bad
        p.dq_, p.dk_, p.dv_ = p.q.cuda(), p.k.cuda(), p.v.cuda()
        _, dk, dv = p.backward(o.float().cuda(), l.float().cuda())
        same(dk[later], want[1][later], tol[1][later], f"dk, {which}")
        same(dv[later], want[2][later], tol[2][later], f"dv, {which}")
        assert not bool(torch.isfinite(dk[:n + shift + 1, 0]).all())
    p.close()
