"""Attention over packed sequences against its definition in 64 bits (tests/seq_util.py, which also
derives the tolerances), forward and backward, through the C ABI."""
import numpy as np
import pytest
import torch

from seq_util import DTYPES, assert_within, attn_backward, attn_forward

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


class Problem:
    """Random tensors of a packed batch on the host and the device, and a plan for them."""

    def __init__(self, dnb, dtype, q_lengths, k_lengths, heads, kv_heads, dim, causal, capacity=None, seed=0, scale=0.0, packed=False):
        self.dnb, self.dt, self.causal, self.scale = dnb, DTYPES[dtype], causal, scale
        gen = torch.Generator().manual_seed(seed + sum(q_lengths) + 7 * sum(k_lengths) + dim)
        rand = lambda *s: torch.randn(s, generator=gen).to(self.dt)
        n = len(q_lengths)
        self.qo = [0] + [int(x) for x in np.cumsum(q_lengths)]
        self.ko = [0] + [int(x) for x in np.cumsum(capacity or k_lengths)]
        self.kl = list(k_lengths) if capacity else None
        rq, rk = self.qo[-1], self.ko[-1]
        self.q, self.dout = rand(rq, heads, dim), rand(rq, heads, dim)
        self.k, self.v = rand(rk, kv_heads, dim), rand(rk, kv_heads, dim)
        if capacity:  # what a cache holds past a sequence's length must not matter
            for s in range(n):
                self.k[self.ko[s] + k_lengths[s]:self.ko[s + 1]] = float("nan")
                self.v[self.ko[s] + k_lengths[s]:self.ko[s + 1]] = float("inf")
        st = dict(q_stride=0, k_stride=0, v_stride=0)
        self.packed = packed and rq == rk
        if self.packed:  # q, k and v side by side in the rows of one matrix
            width = (heads + 2 * kv_heads) * dim
            self.rows = torch.cat([t.reshape(rq, -1) for t in (self.q, self.k, self.v)], 1).cuda()
            self.dq_, self.dk_, self.dv_ = self.rows.split([heads * dim, kv_heads * dim, kv_heads * dim], 1)
            st = dict(q_stride=width, k_stride=width, v_stride=width)
        else:
            self.dq_, self.dk_, self.dv_ = self.q.cuda(), self.k.cuda(), self.v.cuda()
        self.o_ = (ints(self.qo), ints(self.ko), None if self.kl is None else ints(self.kl))
        self.plan = dnb.dnb_attn_create(heads, kv_heads, dim, n, rq, rk, dtype=dnb.DNB_F32 if dtype == "f32" else dnb.DNB_BF16,
                                        causal=causal, scale=scale, **st)
        self.ws = torch.full((max(16, dnb.dnb_attn_workspace_bytes(self.plan)),), 255, dtype=torch.uint8, device="cuda")  # NaN

    def forward(self):
        out = torch.full(self.q.shape, float("nan"), dtype=self.dt, device="cuda")
        lse = torch.full((self.q.shape[1], self.q.shape[0]), float("nan"), device="cuda")
        self.dnb.dnb_attn_forward(self.plan, self.dq_, self.dk_, self.dv_, *self.o_, out, lse, self.ws)
        torch.cuda.synchronize()
        return out, lse

    def backward(self, out, lse):
        dout = self.dout.cuda()
        if self.packed:
            g = torch.full_like(self.rows, float("nan"))
            dq, dk, dv = g.split([t.shape[1] for t in (self.dq_, self.dk_, self.dv_)], 1)
        else:
            dq, dk, dv = (torch.full(t.shape, float("nan"), dtype=self.dt, device="cuda") for t in (self.q, self.k, self.v))
        self.dnb.dnb_attn_backward(self.plan, self.dq_, self.dk_, self.dv_, out, lse, dout, *self.o_, dq, dk, dv, self.ws)
        torch.cuda.synchronize()
        return dq.reshape(self.q.shape), dk.reshape(self.k.shape), dv.reshape(self.v.shape)

    def oracle(self):
        return attn_forward(self.q, self.k, self.v, self.qo, self.ko, self.kl, self.causal, self.scale)

    def check_forward(self):
        out, lse = self.forward()
        o, l, to, tl = self.oracle()
        assert_within(out, o, to, "out")
        assert_within(lse, l, tl, "lse")

    def check_backward(self):
        # from the definition's own out and lse, so that only this pass is measured
        o, l, _, _ = self.oracle()
        out, lse = o.to(self.dt), l.float()
        got = self.backward(out.cuda(), lse.cuda())
        want, tol = attn_backward(self.q, self.k, self.v, out, lse, self.dout, self.qo, self.ko, self.kl, self.causal, self.scale)
        for g, w, t, name in zip(got, want, tol, ("dq", "dk", "dv")):
            assert_within(g, w, t, name)

    def close(self):
        self.dnb.dnb_attn_destroy(self.plan)


# (query lengths, key lengths): one token, tile borders, empty sequences, more queries than keys
PACKED = {"one": ([1], [1]), "borders": ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]), "long": ([300, 1, 129], [300, 1, 129]),
          "empty": ([0, 5, 0, 70, 0], [0, 5, 0, 70, 0]), "chunks": ([7, 40, 1, 90], [200, 40, 131, 95]),
          "more_queries": ([9, 150, 33], [4, 100, 0]), "no_keys": ([40, 3], [0, 0])}


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("lengths", PACKED, ids=list(PACKED))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_sequences(dnb, dtype, lengths, causal):
    p = Problem(dnb, dtype, *PACKED[lengths], 4, 2, 64, causal)
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 8), (2, 2, 32), (7, 1, 40), (6, 2, 64), (8, 8, 72), (3, 3, 80), (14, 2, 96), (9, 3, 104),
                                                (8, 1, 128), (32, 8, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_and_head_dimensions(dnb, dtype, heads, kv_heads, dim):
    p = Problem(dnb, dtype, [77, 20, 140], [77, 50, 140], heads, kv_heads, dim, True)
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 32), (4, 4, 64), (32, 8, 128), (7, 1, 40), (24, 3, 80), (16, 2, 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_over_a_cache(dnb, dtype, heads, kv_heads, dim):
    """One query a request; lengths around the 32 keys of a unit of work, an empty one, and a long one
    that many waves share.  Rows of the cache past a length hold NaN and infinities."""
    ks = [1, 31, 32, 33, 0, 64, 65, 1000, 3000, 2]
    p = Problem(dnb, dtype, [1] * len(ks), ks, heads, kv_heads, dim, True, capacity=[k + 40 for k in ks])
    assert dnb.dnb_attn_workspace_bytes(p.plan) > 4 * heads * len(ks) + 4096   # the form that splits the keys
    p.check_forward()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_requests(dnb, dtype):
    """More sequences than a wave looks at in one step; some without queries, some without keys."""
    r = np.random.default_rng(5)
    q, k = r.integers(0, 4, 150), r.integers(0, 90, 150)
    p = Problem(dnb, dtype, [int(x) for x in q], [int(x) for x in k], 4, 2, 32, True)
    p.check_forward()
    p.check_backward()
    p.close()
    p = Problem(dnb, dtype, [int(x) + 60 for x in q], [int(x) + 60 for x in k], 2, 1, 32, False)
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_drafted_tokens_a_request(dnb, dtype, causal):
    """Several queries a request, still fewer rows than a tile on average, over more than one tile in one."""
    p = Problem(dnb, dtype, [5, 1, 0, 40, 3, 2], [70, 1, 9, 300, 2, 0], 8, 4, 64, causal, capacity=[80, 1, 20, 333, 2, 5])
    p.check_forward()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_one_product(dnb, dtype):
    """q, k and v, and their gradients, side by side in the rows of one matrix."""
    p = Problem(dnb, dtype, [50, 130, 3], [50, 130, 3], 6, 2, 48, True, packed=True, scale=0.3)
    assert p.packed
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unused_room_gets_zero_gradients_and_foreign_rows_stay(dnb, dtype):
    p = Problem(dnb, dtype, [40, 20], [33, 20], 2, 1, 32, True, capacity=[70, 200])
    o, l, _, _ = p.oracle()
    _, dk, dv = p.backward(o.to(p.dt).cuda(), l.float().cuda())
    for d in (dk, dv):
        assert bool((d[33:70] == 0).all()) and bool((d[90:270] == 0).all())
        assert bool(torch.isfinite(d.float()).all())
    p.check_backward()
    # rows outside every sequence are not written
    p.o_ = (ints([3, 20, 50]), ints([2, 60, 250]), ints([33, 20]))
    out, lse = p.forward()
    assert bool(torch.isnan(out[:3].float()).all()) and bool(torch.isnan(out[50:].float()).all())
    assert bool(torch.isnan(lse[:, :3]).all()) and bool(torch.isnan(lse[:, 50:]).all())
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_infinite_ones(dnb, dtype):
    """Scores far beyond what exp takes; keys of minus infinity that a query has to ignore."""
    p = Problem(dnb, dtype, [70], [70], 2, 2, 32, True, scale=40.0)
    p.check_forward()
    p.close()
    p = Problem(dnb, dtype, [20], [100], 1, 1, 32, False)
    p.q = p.q.abs() + 0.5
    p.k[10:90] = -float("inf")   # scores of -inf
    p.dq_, p.dk_ = p.q.cuda(), p.k.cuda()
    out, lse = p.forward()
    keep = list(range(10)) + list(range(90, 100))
    o, l, to, tl = attn_forward(p.q, p.k[keep], p.v[keep], [0, 20], [0, 20], None, False)
    assert_within(out, o, to, "out")
    assert_within(lse, l, tl, "lse")
    p.close()


def test_hidden_keys_that_are_nan_do_not_reach_earlier_queries(dnb):
    """Keys (not values) of NaN behind the causal mask: their scores are replaced, not added to."""
    p = Problem(dnb, "bf16", [64], [64], 2, 2, 64, True)
    p.k[50:] = float("nan")
    p.dk_ = p.k.cuda()
    out, _ = p.forward()
    o, _, to, _ = attn_forward(p.q[:50], p.k[:50], p.v[:50], [0, 50], [0, 50], None, True)
    assert_within(out[:50], o, to, "out")
    assert bool(torch.isnan(out[50:].float()).all())
    p.close()


def test_offsets_past_32_bits(dnb):
    """Keys whose elements lie beyond 2^31: rows 2^22 elements apart."""
    stride, rows = 1 << 22, 600
    buf = torch.empty(stride * rows, dtype=torch.bfloat16, device="cuda")
    for lengths, form in (([1, 1], "token"), ([100, 300], "tile")):
        p = Problem(dnb, "bf16", lengths, [100, 500], 2, 1, 64, True)
        k = buf.as_strided((rows, 64), (stride, 1))
        v = buf[64:].as_strided((rows, 64), (stride, 1))
        k.copy_(p.dk_.reshape(rows, 64))
        v.copy_(p.dv_.reshape(rows, 64))
        dnb.dnb_attn_destroy(p.plan)
        p.plan = dnb.dnb_attn_create(2, 1, 64, 2, sum(lengths), rows, causal=True, k_stride=stride, v_stride=stride)
        p.dk_, p.dv_ = k, v
        p.check_forward()
        p.close()
    del buf


@pytest.mark.parametrize("token", [True, False], ids=["token", "tile"])
def test_offsets_outside_the_tensors_are_cut_to_them(dnb, token):
    q = [1, 1, 1] if token else [40, 60, 50]
    p = Problem(dnb, "bf16", q, [50, 60, 70], 4, 2, 64, True)
    good = p.o_
    a = p.forward()[0]
    big = 2 ** 31 - 1
    p.o_ = (torch.cat([ints([-5]), good[0][1:-1], ints([big])]), torch.cat([ints([-big]), good[1][1:-1], ints([big])]), None)
    assert torch.equal(a, p.forward()[0])
    p.o_ = (good[0], good[1], ints([big, -big, 10 ** 6]))
    b = p.forward()[0]
    assert torch.equal(a[:q[0]], b[:q[0]]) and bool((b[q[0]:q[0] + q[1]] == 0).all()) and torch.equal(a[q[0] + q[1]:], b[q[0] + q[1]:])
    p.o_ = (ints([9, 2, big, -7]), ints([100, -3, 50, 7]), ints([big, 5, -1]))   # what comes out is undefined
    p.forward()
    p.backward(*p.forward())
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("token", [True, False], ids=["token", "tile"])
def test_repeats_bit_for_bit(dnb, dtype, token):
    q = [1] * 6 if token else [300, 40]
    k = [900, 5, 77, 300, 1, 64] if token else [500, 40]
    p = Problem(dnb, dtype, q, k, 8, 2, 64, True)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    for _ in range(3):
        p.ws.fill_(255)
        o, l = p.forward()
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    p.close()


def test_gradients_against_differences(dnb):
    """The whole chain in fp32: <gradient, direction> against central differences of the definition."""
    p = Problem(dnb, "f32", [33, 90], [60, 90], 4, 2, 40, True)
    grads = p.backward(*p.forward())
    gen = torch.Generator().manual_seed(3)
    loss = lambda q, k, v: float((attn_forward(q, k, v, p.qo, p.ko, None, True)[0] * p.dout.double()).sum())
    x = [t.double() for t in (p.q, p.k, p.v)]
    for i, name in enumerate(("dq", "dk", "dv")):
        step = torch.randn(x[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * step, x[i] - h * step
        want = (loss(*up) - loss(*down)) / (2 * h)
        got = float((grads[i].double().cpu() * step).sum())
        # fp32 gradients (relative 2^-24 times sums of some hundred terms) and differences of order h^2
        assert abs(got - want) <= 1e-4 * float((grads[i].double().cpu() * step).abs().sum()) ** 0.5 + 1e-4 * abs(want), (name, got, want)
    p.close()


@pytest.mark.parametrize("token", [True, False], ids=["token", "tile"])
def test_in_a_graph_and_on_another_stream(dnb, token):
    """Captured once and replayed on new values, with eager work between the replays."""
    q = [1, 1, 1] if token else [100, 40, 7]
    p = Problem(dnb, "bf16", q, [200, 64, 7], 4, 2, 64, True)
    out = torch.empty(p.q.shape, dtype=p.dt, device="cuda")
    lse = torch.empty((4, p.q.shape[0]), device="cuda")
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


# few rows and long keys: the work is split over the keys, forward and for dq
SPLIT = {"one": ([1], [3000]), "prompt": ([700], [700]), "chunks": ([40, 3, 100, 0, 1], [900, 1200, 700, 50, 2000]),
         "more_queries": ([90, 700], [30, 690]), "empty": ([5, 0, 33, 2], [0, 900, 3000, 1])}


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("lengths", SPLIT, ids=list(SPLIT))
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 128), (6, 2, 64), (7, 1, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows_over_long_keys(dnb, dtype, heads, kv_heads, dim, lengths, causal):
    q, k = SPLIT[lengths]
    p = Problem(dnb, dtype, q, k, heads, kv_heads, dim, causal, capacity=[x + 9 for x in k])
    p.check_forward()
    p.check_backward()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows_over_long_keys_repeat_and_offsets_are_cut(dnb, dtype):
    p = Problem(dnb, dtype, [20, 60, 5], [700, 1500, 900], 4, 2, 96, True)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    for _ in range(3):
        p.ws.fill_(255)
        o, l = p.forward()
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    big = 2 ** 31 - 1
    p.o_ = (torch.cat([ints([-5]), p.o_[0][1:-1], ints([big])]), torch.cat([ints([-big]), p.o_[1][1:-1], ints([big])]), None)
    o, l = p.forward()
    assert torch.equal(o, out) and all(torch.equal(a, b) for a, b in zip(p.backward(o, l), grads))
    p.o_ = (ints([9, 2, big, -7]), ints([100, -3, 50, 7]), ints([big, 5, -1]))   # what comes out is undefined
    p.backward(*p.forward())
    p.close()
