"""Norms of queries and keys with their rotation, and the form that writes the pages of a cache, against 64 bits.

Rounding: x^2 summed over up to 256 values in fp32 is off by at most 256 steps of 2^-24 of the sum, of which the root keeps half; the root,
division, products with the weight and factor, the angle's fraction of a turn (2^-25 of a turn, 2 pi of that in radians), cosine and
sine and the rotation's two products and sum add some 20 steps of 2^-24 of |a| + |b|; then comes the type's own rounding."""
import math

import numpy as np
import pytest
import torch

from paged_util import LAYOUTS, Cache, ints, offsets
from seq_util import DTYPES, assert_within, half_step

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def turns_of(rotary):
    return 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1)) / (2 * math.pi)


def spin(x, positions, turns, rotary, interleaved, sign=1.0):
    """(turned x, sum of magnitudes of each value's terms)"""
    if rotary == 0:
        return x.clone(), x.abs()
    angle = 2 * math.pi * positions.double()[:, None, None] * turns
    c, s = torch.cos(angle), sign * torch.sin(angle)
    at = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    y, size = x.clone(), x.abs()
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
    return y, size


def forward(x, w, positions, turns, rotary, interleaved, eps, factor, dtype):
    """x (rows, heads, dim) in 64 bits -> (y, bound)"""
    n = x if w is None else x / torch.sqrt(x.square().mean(2, keepdim=True) + eps) * w.double()
    y, size = spin(n, positions, turns, rotary, interleaved)
    if rotary:
        y[..., :rotary], size[..., :rotary] = y[..., :rotary] * factor, size[..., :rotary] * abs(factor)
    e = F * (40 + (x.shape[2] if w is not None else 0))
    return y, half_step(dtype) * y.abs() + e * size


def backward(x, w, dy, positions, turns, rotary, interleaved, eps, factor, dtype):
    dn, size = spin(dy, positions, turns, rotary, interleaved, -1.0)
    if rotary:
        dn[..., :rotary], size[..., :rotary] = dn[..., :rotary] * factor, size[..., :rotary] * abs(factor)
    d = x.shape[2]
    if w is None:
        return dn, half_step(dtype) * dn.abs() + 40 * F * size, None, None
    w = w.double()
    inv = 1 / torch.sqrt(x.square().mean(2, keepdim=True) + eps)
    u = x * inv
    t = dn * w
    dx = inv * (t - u * (t * u).mean(2, keepdim=True))
    mag = inv * (size * w.abs() + u.abs() * (size * w.abs() * u.abs()).mean(2, keepdim=True))
    e = F * (60 + 2 * d)
    n = x.shape[0] * x.shape[1]
    return dx, half_step(dtype) * dx.abs() + e * mag, (dn * u).sum((0, 1)), F * (60 + d + n) * (size * u.abs()).sum((0, 1))


class Case:
    def __init__(self, dnb, rows, hq, hk, dim, rotary, dtype, interleaved=False, norm="both", factor=1.0, far=100000, eps=1e-6, packed=True, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.dt, self.rows, self.hq, self.hk, self.dim, self.rotary = DTYPES[dtype], rows, hq, hk, dim, rotary
        self.interleaved, self.factor, self.eps = interleaved, factor, eps
        width = (hq + 2 * hk) * dim if packed else 0
        self.x = (torch.randn(rows, (hq + 2 * hk) * dim, generator=gen) * 1.5).to(self.dt)
        self.w_q = 1 + 0.2 * torch.randn(dim, generator=gen) if norm in ("both", "q") else None
        self.w_k = 1 + 0.2 * torch.randn(dim, generator=gen) if norm in ("both", "k") else None
        self.positions = torch.randint(-far, far, (rows,), generator=gen, dtype=torch.int32)
        self.turns = turns_of(rotary)
        self.gpu = self.x.cuda()
        cut = [hq * dim, hk * dim, hk * dim]
        views = self.gpu.split(cut, 1)
        self.q, self.k, self.v = views if packed else (t.contiguous() for t in views)
        self.layout = dnb.dnb_qk_layout(rows, hq, hk, dim, rotary, dnb.DNB_ROPE_INTERLEAVED if interleaved else dnb.DNB_ROPE_HALF,
                                        dtype=dnb.DNB_F32 if dtype == "f32" else dnb.DNB_BF16, eps=eps, factor=factor, q_stride=width, k_stride=width,
                                        v_stride=width)
        up = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.gw_q, self.gw_k, self.gpos, self.gturns = up(self.w_q), up(self.w_k), up(self.positions), up(self.turns)

    def heads(self, which):
        a, n = (0, self.hq) if which == "q" else (self.hq, self.hk) if which == "k" else (self.hq + self.hk, self.hk)
        return self.x[:, a * self.dim:(a + n) * self.dim].double().reshape(self.rows, n, self.dim)

    def want(self, which, positions=None):
        w = self.w_q if which == "q" else self.w_k
        return forward(self.heads(which), w, self.positions if positions is None else positions, self.turns, self.rotary, self.interleaved, self.eps,
                       self.factor, self.dt)

    def out(self, n, value=5.0):
        return torch.full((self.rows, n, self.dim), value, dtype=self.dt, device="cuda")


SHAPES = [(1, 1, 1, 128, 128, False), (3, 32, 8, 128, 128, False), (70, 5, 3, 128, 64, True), (9, 7, 1, 64, 64, True), (33, 4, 2, 80, 40, False),
          (20, 15, 5, 80, 40, True), (17, 3, 2, 32, 32, False), (5, 2, 2, 256, 256, False), (4, 3, 1, 256, 128, True), (11, 2, 1, 20, 12, False),
          (13, 3, 3, 6, 6, False), (6, 2, 1, 250, 250, False), (8, 2, 1, 254, 30, True), (7, 1, 1, 2, 2, False), (12, 2, 1, 96, 0, False),
          (300, 12, 4, 96, 96, False), (5, 200, 30, 64, 64, False), (9, 4, 2, 8, 8, True), (6, 1, 3, 16, 8, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_forward_and_gradients(dnb, dtype, packed, shape):
    rows, hq, hk, dim, rotary, inter = shape
    c = Case(dnb, rows, hq, hk, dim, rotary, dtype, inter, factor=1.25, packed=packed)
    yq, yk = c.out(hq), c.out(hk)
    if c.k.data_ptr() % 16:   # keys that begin off 16 bytes in their rows are refused, as every tensor there
        with pytest.raises(dnb.DnbError) as refused:
            dnb.dnb_op_qk_rope_forward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, yq, yk)
        assert refused.value.status == dnb.DNB_E_ALIGN
        return
    dnb.dnb_op_qk_rope_forward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, yq, yk)
    assert_within(yq, *c.want("q"), "q")
    assert_within(yk, *c.want("k"), "k")
    gen = torch.Generator().manual_seed(9)
    dyq, dyk = (torch.randn(rows, n, dim, generator=gen).to(c.dt) for n in (hq, hk))
    dx = torch.full_like(c.gpu, 3.0)
    dq, dk = (dx[:, :hq * dim], dx[:, hq * dim:(hq + hk) * dim]) if packed else (torch.empty_like(c.q), torch.empty_like(c.k))
    dwq, dwk = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    scratch = torch.full((dnb.dnb_op_qk_rope_scratch_bytes(c.layout),), 0xff, dtype=torch.uint8, device="cuda")
    dnb.dnb_op_qk_rope_backward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, dyq.cuda(), dyk.cuda(), dq, dk, dwq, dwk, scratch)
    for which, dy, got, dw, w in (("q", dyq, dq, dwq, c.w_q), ("k", dyk, dk, dwk, c.w_k)):
        want, tol, wwant, wtol = backward(c.heads(which), w, dy.double(), c.positions, c.turns, rotary, inter, c.eps, c.factor, c.dt)
        assert_within(got.reshape(rows, -1, dim), want, tol, "d" + which)
        assert_within(dw, wwant, wtol, "dw_" + which)
    if packed:
        assert (dx[:, (hq + hk) * dim:] == 3).all()


@pytest.mark.parametrize("norm", ["none", "q", "k"])
def test_heads_that_are_not_normed(dnb, norm):
    c = Case(dnb, 21, 6, 2, 64, 64, "f32", norm=norm)
    yq, yk = c.out(6), c.out(2)
    dnb.dnb_op_qk_rope_forward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, yq, yk)
    assert_within(yq, *c.want("q"), "q")
    assert_within(yk, *c.want("k"), "k")
    dy = torch.randn(21, 6, 64, generator=torch.Generator().manual_seed(2)), torch.randn(21, 2, 64, generator=torch.Generator().manual_seed(3))
    dq, dk = torch.empty_like(c.q), torch.empty_like(c.k)
    dq, dk = (torch.empty_like(c.gpu)[:, :6 * 64], torch.empty_like(c.gpu)[:, 6 * 64:8 * 64])
    dws = [None if w is None else torch.empty(64, device="cuda") for w in (c.w_q, c.w_k)]
    scratch = torch.empty(dnb.dnb_op_qk_rope_scratch_bytes(c.layout), dtype=torch.uint8, device="cuda")
    dnb.dnb_op_qk_rope_backward(c.layout, c.q if norm == "q" else None, c.k if norm == "k" else None, c.gw_q, c.gw_k, c.gpos, c.gturns, dy[0].cuda(),
                                dy[1].cuda(), dq, dk, *dws, scratch)
    for which, d, got, dw, w in (("q", dy[0], dq, dws[0], c.w_q), ("k", dy[1], dk, dws[1], c.w_k)):
        want, tol, wwant, wtol = backward(c.heads(which), w, d.double(), c.positions, c.turns, 64, False, c.eps, c.factor, c.dt)
        assert_within(got.reshape(21, -1, 64), want, tol, "d" + which)
        if w is not None:
            assert_within(dw, wwant, wtol, "dw_" + which)


def test_gradients_against_differences(dnb):
    """In fp32: the loss's change along a direction over a step of 2^-7, centred (error of the third derivative, h^2, and 2^-24 / h)."""
    c = Case(dnb, 5, 2, 1, 16, 16, "f32", packed=False, far=50)
    gen = torch.Generator().manual_seed(4)
    dyq, dyk = torch.randn(5, 2, 16, generator=gen).cuda(), torch.randn(5, 1, 16, generator=gen).cuda()
    dq, dk, dwq, dwk = torch.empty_like(c.q), torch.empty_like(c.k), torch.empty(16, device="cuda"), torch.empty(16, device="cuda")
    scratch = torch.empty(dnb.dnb_op_qk_rope_scratch_bytes(c.layout), dtype=torch.uint8, device="cuda")
    dnb.dnb_op_qk_rope_backward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, dyq, dyk, dq, dk, dwq, dwk, scratch)

    def loss(q, k, wq, wk):
        yq, yk = c.out(2), c.out(1)
        dnb.dnb_op_qk_rope_forward(c.layout, q, k, wq, wk, c.gpos, c.gturns, yq, yk)
        return float((yq.double() * dyq).sum() + (yk.double() * dyk).sum())
    h = 2.0 ** -7
    leaves, grads = [c.q, c.k, c.gw_q, c.gw_k], [dq, dk, dwq, dwk]
    for i, (leaf, g) in enumerate(zip(leaves, grads)):
        d = torch.randn(leaf.shape, generator=gen).cuda()
        up, down = list(leaves), list(leaves)
        up[i], down[i] = leaf + h * d, leaf - h * d
        slope = (loss(*up) - loss(*down)) / (2 * h)
        along = float((g.double() * d.double()).sum())
        size = float((g.double() * d.double()).abs().sum())
        assert abs(slope - along) <= 0.02 * size + 1e-3, i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dnb, dtype):
    c = Case(dnb, 40, 8, 2, 128, 128, dtype)
    width = c.gpu.shape[1]
    layout = dnb.dnb_qk_layout(40, 8, 2, 128, 128, dtype=c.layout.dtype, q_stride=width, k_stride=width, q_out_stride=width, k_out_stride=width)
    v = c.v.clone()
    dnb.dnb_op_qk_rope_forward(layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, c.q, c.k)
    assert_within(c.q.reshape(40, 8, 128), *c.want("q"), "q")
    assert_within(c.k.reshape(40, 2, 128), *c.want("k"), "k")
    assert torch.equal(v, c.v)
    dx = torch.randn(40, width, generator=torch.Generator().manual_seed(1)).to(c.dt)
    g = dx.cuda()
    x = c.x.cuda()
    q, k, dq, dk = x[:, :1024], x[:, 1024:1280], g[:, :1024], g[:, 1024:1280]
    dw = [torch.empty(128, device="cuda") for _ in range(2)]
    scratch = torch.empty(dnb.dnb_op_qk_rope_scratch_bytes(layout), dtype=torch.uint8, device="cuda")
    dnb.dnb_op_qk_rope_backward(layout, q, k, c.gw_q, c.gw_k, c.gpos, c.gturns, dq, dk, dq, dk, *dw, scratch)
    want, tol, _, _ = backward(c.heads("q"), c.w_q, dx[:, :1024].double().reshape(40, 8, 128), c.positions, c.turns, 128, False, c.eps, 1.0, c.dt)
    assert_within(dq.reshape(40, 8, 128), want, tol, "dq")


def test_no_rows(dnb):
    """Gradients of weights are zero then, and only queries may be there."""
    layout = dnb.dnb_qk_layout(0, 4, 2, 64, 64)
    w = torch.ones(64, device="cuda")
    dw = [torch.full((64,), 5.0, device="cuda") for _ in range(2)]
    dnb.dnb_op_qk_rope_backward(layout, None, None, w, w, None, None, None, None, None, None, *dw, None)
    assert (dw[0] == 0).all() and (dw[1] == 0).all()
    c = Case(dnb, 10, 3, 0, 64, 64, "bf16")
    y = c.out(3)
    dnb.dnb_op_qk_rope_forward(c.layout, c.q, None, c.gw_q, None, c.gpos, c.gturns, y, None)
    assert_within(y, *c.want("q"), "q")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_repeat_bit_for_bit_in_a_graph(dnb, dtype):
    c = Case(dnb, 3001, 16, 4, 128, 128, dtype)
    dyq, dyk = torch.randn(3001, 16, 128, device="cuda").to(c.dt), torch.randn(3001, 4, 128, device="cuda").to(c.dt)
    scratch = torch.empty(dnb.dnb_op_qk_rope_scratch_bytes(c.layout), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(c.gpu)
    dq, dk = dx[:, :2048], dx[:, 2048:2560]
    dw = [torch.empty(128, device="cuda") for _ in range(2)]

    def call():
        dnb.dnb_op_qk_rope_backward(c.layout, c.q, c.k, c.gw_q, c.gw_k, c.gpos, c.gturns, dyq, dyk, dq, dk, *dw, scratch)
    call()
    first = [t.clone() for t in (dq, dk, *dw)]
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            call()
    for _ in range(3):
        for t in (dx, *dw, scratch):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (dq, dk, *dw)))


# ---------------------------------------------------------------- the pages of a cache

def append(dnb, c, cache, new, positions=None, q_offsets=None, lengths=None, table=None):
    k, v = cache.to_gpu()
    before = k.clone(), v.clone()
    out = c.out(c.hq)
    dnb.dnb_op_paged_append(c.layout, cache.layout_of(dnb), c.q if c.hq else None, c.k, c.v, c.gw_q, c.gw_k, positions, c.gturns,
                            ints(offsets(new)) if q_offsets is None else q_offsets, ints(cache.lengths) if lengths is None else lengths,
                            ints(cache.table) if table is None else table, out, k, v)
    torch.cuda.synchronize()
    return out, k, v, before


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("page,new,lengths", [(16, [1, 1, 1], [1, 17, 300]), (8, [40, 1, 0, 9], [40, 100, 5, 30]), (1, [3], [9]),
                                              (64, [0, 0, 70, 0, 1], [0, 3, 200, 0, 64]), (32, [1] * 130, [i % 50 + 1 for i in range(130)])])
def test_append(dnb, dtype, layout, page, new, lengths):
    """Rows of the pools that no new token has are not touched, q's rows behind the last sequence neither."""
    kv, dim = 2, 64
    cache = Cache(lengths, page, kv, dim, DTYPES[dtype], layout)
    c = Case(dnb, sum(new) + 3, 6, kv, dim, dim, dtype)
    out, k, v, before = append(dnb, c, cache, new)
    n = sum(new)
    place = torch.cat([torch.arange(b - a, b) for a, b in zip(new, lengths)])
    pos = torch.cat([place, torch.zeros(3, dtype=place.dtype)])
    want, tol = c.want("q", pos)
    assert_within(out[:n], want[:n], tol[:n], "q")
    assert (out[n:] == 5).all()
    seq = np.repeat(np.arange(len(new)), new)
    page_of, row = cache.table[seq, place.numpy() // page].astype(np.int64), place.numpy() % page
    wk, tk = c.want("k", pos)
    view = (lambda t: t.transpose(1, 2)) if layout == "heads" else (lambda t: t)
    assert_within(view(k)[page_of, row], wk[:n], tk[:n], "k")
    assert torch.equal(view(v)[page_of, row].cpu().double(), c.heads("v")[:n])
    for got, was in ((k, before[0]), (v, before[1])):
        got, was = view(got).clone(), view(was)
        got[page_of, row] = was[page_of, row]
        assert torch.equal(torch.nan_to_num(got, nan=77.0), torch.nan_to_num(was, nan=77.0))


def test_append_at_given_positions_and_bad_places(dnb):
    """Given positions turn; pages outside the pool, tokens before the first and past the table are not written."""
    cache = Cache([40, 20, 3], 8, 2, 32, torch.float32)
    c = Case(dnb, 30, 4, 2, 32, 32, "f32")
    table = cache.table.copy()
    table[1, 1] = cache.pages   # tokens 8 to 15 of the second
    table[1, 2] = -7            # 16 to 19
    out, k, v, before = append(dnb, c, cache, None, c.gpos, ints([0, 10, 24, 30]), ints([40, 20, 3]), ints(table))
    assert_within(out, *c.want("q"), "q")
    wk, tk = c.want("k")
    k, v, bk, bv = (t.cpu() for t in (k, v, *before))
    written = np.zeros((cache.pages, 8), dtype=bool)
    for row in range(30):
        s = 0 if row < 10 else 1 if row < 24 else 2
        first, n, length = ((0, 10, 40), (10, 14, 20), (24, 6, 3))[s]
        j = row - first + length - n
        p = table[s, j // 8] if j >= 0 else -1
        if 0 <= p < cache.pages:
            written[p, j % 8] = True
            assert_within(k[p, j % 8], wk[row], tk[row], "k")
            assert torch.equal(v[p, j % 8].double(), c.heads("v")[row])
    rest = torch.tensor(~written)
    assert written.sum() == 10 + 2 + 3
    assert torch.equal(torch.nan_to_num(k[rest]), torch.nan_to_num(bk[rest])) and torch.equal(torch.nan_to_num(v[rest]), torch.nan_to_num(bv[rest]))


def test_append_without_queries_norm_or_turning(dnb):
    cache = Cache([20, 9], 16, 3, 40, torch.bfloat16)
    c = Case(dnb, 12, 0, 3, 40, 0, "bf16", norm="none")
    _, k, v, _ = append(dnb, c, cache, [10, 2])
    for row, (s, j) in enumerate([(0, 10 + i) for i in range(10)] + [(1, 7), (1, 8)]):
        p = int(cache.table[s, j // 16])
        assert torch.equal(k[p, j % 16].cpu().double(), c.heads("k")[row]) and torch.equal(v[p, j % 16].cpu().double(), c.heads("v")[row])


@pytest.mark.parametrize("n", [64, 65, 4097, 9000])
def test_append_to_many_sequences(dnb, n):
    lengths = [1 + i % 5 if i % 7 else 0 for i in range(n)]
    new = [min(v, i % 2 + 1) for i, v in enumerate(lengths)]
    cache = Cache(lengths, 8, 1, 8, torch.float32)
    c = Case(dnb, sum(new), 1, 1, 8, 8, "f32")
    out, k, v, _ = append(dnb, c, cache, new)
    place = torch.cat([torch.arange(b - a, b) for a, b in zip(new, lengths)])
    assert_within(out, *c.want("q", place), "q")
    seq = np.repeat(np.arange(n), new)
    assert_within(k[cache.table[seq, place.numpy() // 8].astype(np.int64), place.numpy() % 8], *c.want("k", place), "k")
