"""The norms around a block against their definition in 64 bits, gradients by automatic differentiation of
it, through the C ABI.

Tolerances: sums of width terms in fp32, pairwise over threads: relative (log2(width) + 16) 2^-24 of the
sums of magnitudes; one rounding of each result to its type.  Column sums add rows: (rows + 16) 2^-24."""
import math

import pytest
import torch

from seq_util import DTYPES, assert_within, half_step

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


def make(dnb, dtype, rows, width, gate, post, seed=0):
    dt = DTYPES[dtype]
    gen = torch.Generator().manual_seed(seed + rows + width)
    rand = lambda *s: torch.randn(s, generator=gen)
    p = {n: rand(rows, width).to(dt) for n in ("b", "r", "dh", "dy")}
    p["w_pre"] = 1 + 0.2 * rand(width)
    p["w_post"] = 1 + 0.2 * rand(width) if post else None
    p["gate"] = {"none": None, "vector": rand(width), "full": torch.sigmoid(rand(rows, width)).to(dt)}[gate]
    kind = {"none": dnb.DNB_GATE_NONE, "vector": dnb.DNB_GATE_VECTOR, "full": dnb.DNB_GATE_FULL}[gate]
    return p, kind, dnb.DNB_F32 if dtype == "f32" else dnb.DNB_BF16


def unit(t, eps):
    return t / torch.sqrt(t.square().mean(1, keepdim=True) + eps)


def forward(p, scale, eps):
    b, r = p["b"].double(), p["r"].double()
    branch = b if p["w_post"] is None else unit(b, eps) * p["w_post"].double()
    g = 1.0 if p["gate"] is None else p["gate"].double()
    h = scale * r + g * branch
    return h, unit(h, eps) * p["w_pre"].double(), (scale * r).abs() + (g * branch).abs()


def cuda(t):
    return None if t is None else t.cuda()


SHAPES = [(1, 8), (3, 64), (16, 4096), (7, 512), (5, 520), (9, 1024), (2, 1032), (6, 2048), (300, 2208), (4, 8192), (3, 8200), (2, 16384), (1500, 72)]


@pytest.mark.parametrize("gate,post", [("none", True), ("vector", True), ("full", True), ("none", False), ("vector", False), ("full", False)])
@pytest.mark.parametrize("rows,width", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forward_and_backward(dnb, dtype, rows, width, gate, post):
    p, kind, code = make(dnb, dtype, rows, width, gate, post)
    dt, scale, eps = DTYPES[dtype], 0.7071, 1e-6
    r = half_step(dt)
    d = {n: cuda(t) for n, t in p.items()}
    new = lambda like: None if like is None else torch.full_like(like, float("nan"))
    h_new, y = new(d["b"]), new(d["b"])
    dnb.dnb_op_norm_residual_forward(d["b"], d["r"], d["w_post"], d["gate"], d["w_pre"], h_new, y, rows, width, scale, eps, kind, code)
    h, yy, size = forward(p, scale, eps)
    f = (math.log2(width) + 16) * F
    inv = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    assert_within(h_new, h, f * size + r * h.abs(), "h_new")
    # an error e of h is e / rms in y, and of every h together moves the rms by no more than its mean square
    wide = torch.sqrt((f * size).square().mean(1, keepdim=True))
    assert_within(y, yy, inv * p["w_pre"].double().abs() * (f * size + h.abs() * inv * wide) + f * yy.abs() + r * yy.abs(), "y")

    # backward, at the h that the program holds: rounded
    hh = h.to(dt)
    out = {n: new(d[k]) for n, k in (("db", "b"), ("dr", "b"), ("dw_post", "w_post"), ("dgate", "gate"), ("dw_pre", "w_pre"))}
    scratch = torch.full((max(16, dnb.dnb_op_norm_residual_scratch_bytes(rows, width, kind)),), 255, dtype=torch.uint8, device="cuda")
    dnb.dnb_op_norm_residual_backward(d["b"], hh.cuda(), d["w_post"], d["gate"], d["w_pre"], d["dh"], d["dy"], out["db"], out["dr"],
                                      out["dw_post"], out["dgate"], out["dw_pre"], rows, width, scale, eps, kind, code, scratch)
    leaf = lambda t: None if t is None else t.double().requires_grad_()
    b, res, wp, g, w, at = leaf(p["b"]), leaf(p["r"]), leaf(p["w_post"]), leaf(p["gate"]), leaf(p["w_pre"]), leaf(hh)
    branch = b if wp is None else unit(b, eps) * wp
    hd = scale * res + (branch if g is None else branch * g)
    yd = unit(at, eps) * w
    dat, dw = torch.autograd.grad(yd, (at, w), p["dy"].double())
    leaves = [(n, t) for n, t in (("db", b), ("dr", res), ("dw_post", wp), ("dgate", g)) if t is not None]
    grads = dict(zip([n for n, _ in leaves], torch.autograd.grad(hd, [t for _, t in leaves], p["dh"].double() + dat)))
    # magnitudes of the terms, by the formulas beside the kernel
    H, t = hh.double(), p["dy"].double() * p["w_pre"].double()
    ih = 1 / torch.sqrt(H.square().mean(1, keepdim=True) + eps)
    xh = (H * ih).abs()
    total = p["dh"].double().abs() + ih * (t.abs() + xh * (t.abs() * xh).mean(1, keepdim=True))
    ib = 1 / torch.sqrt(p["b"].double().square().mean(1, keepdim=True) + eps) if post else torch.ones(rows, 1, dtype=torch.float64)
    xb = (p["b"].double() * ib).abs()
    ga = 1.0 if p["gate"] is None else p["gate"].double().abs()
    wpa = 1.0 if not post else p["w_post"].double().abs()
    du = total * ga * wpa
    f2 = 2 * f
    tol = {"dr": f2 * scale * total + r * grads["dr"].abs(),
           "db": f2 * ib * (du + (xb * (du * xb).mean(1, keepdim=True) if post else 0)) + r * grads["db"].abs()}
    fr = f2 + (rows + 16) * F
    if post:
        tol["dw_post"] = fr * (total * ga * xb).sum(0)
    if gate == "vector":
        tol["dgate"] = fr * (total * xb * wpa).sum(0)
    if gate == "full":
        tol["dgate"] = f2 * total * xb * wpa + r * grads["dgate"].abs()
    grads["dw_pre"], tol["dw_pre"] = dw, fr * (p["dy"].double().abs() * xh).sum(0)
    for n in tol:
        assert_within(out[n], grads[n].detach(), tol[n].detach(), n)


def test_gradients_against_differences(dnb):
    """Both norms in fp32 as one function: <gradient, step> against central differences in 64 bits."""
    rows, width, scale, eps = 6, 136, 0.5, 1e-5
    p, kind, code = make(dnb, "f32", rows, width, "vector", True)
    d = {n: cuda(t) for n, t in p.items()}
    h, y = torch.empty_like(d["b"]), torch.empty_like(d["b"])
    dnb.dnb_op_norm_residual_forward(d["b"], d["r"], d["w_post"], d["gate"], d["w_pre"], h, y, rows, width, scale, eps, kind, code)
    g = {n: torch.empty_like(d[n]) for n in ("b", "r", "w_post", "gate", "w_pre")}
    scratch = torch.empty(dnb.dnb_op_norm_residual_scratch_bytes(rows, width, kind), dtype=torch.uint8, device="cuda")
    dnb.dnb_op_norm_residual_backward(d["b"], h, d["w_post"], d["gate"], d["w_pre"], d["dh"], d["dy"], g["b"], g["r"], g["w_post"], g["gate"],
                                      g["w_pre"], rows, width, scale, eps, kind, code, scratch)

    def loss(q):
        hh, yy, _ = forward(q, scale, eps)
        return float((hh * p["dh"].double()).sum() + (yy * p["dy"].double()).sum())

    gen = torch.Generator().manual_seed(9)
    for n in g:
        step = torch.randn(p[n].shape, generator=gen, dtype=torch.float64)
        up, down = ({**{k: None if v is None else v.double() for k, v in p.items()}, n: p[n].double() + s * 1e-5 * step} for s in (1, -1))
        want, terms = (loss(up) - loss(down)) / 2e-5, g[n].double().cpu() * step
        # fp32 gradients: some 100 steps of 2^-24 of their terms; differences: h^2 and 2^-53 / h of a loss of some hundred
        assert abs(float(terms.sum()) - want) <= 100 * F * float(terms.abs().sum()) + 1e-7 * (1 + abs(want)), n


def test_no_rows(dnb):
    """No rows: nothing is written but the column sums, which are zero."""
    p, kind, code = make(dnb, "f32", 1, 64, "vector", True)
    d = {n: cuda(t) for n, t in p.items()}
    dnb.dnb_op_norm_residual_forward(None, None, d["w_post"], d["gate"], d["w_pre"], None, None, 0, 64, 1.0, 1e-6, kind, code)
    out = [torch.full((64,), float("nan"), device="cuda") for _ in range(3)]
    dnb.dnb_op_norm_residual_backward(None, None, d["w_post"], d["gate"], d["w_pre"], None, None, None, None, out[0], out[1], out[2], 0, 64, 1.0,
                                      1e-6, kind, code, None)
    assert all(bool((t == 0).all()) for t in out)


def test_repeats_bit_for_bit_and_in_a_graph(dnb):
    rows, width, scale, eps = 2000, 1536, 0.5, 1e-6
    p, kind, code = make(dnb, "bf16", rows, width, "vector", True)
    d = {n: cuda(t) for n, t in p.items()}
    scratch = torch.empty(dnb.dnb_op_norm_residual_scratch_bytes(rows, width, kind), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(d[n]) for n in ("b", "b", "b", "b", "w_post", "gate", "w_pre")]

    def calls(stream=None):
        h, y, db, dr, dwp, dg, dw = out
        dnb.dnb_op_norm_residual_forward(d["b"], d["r"], d["w_post"], d["gate"], d["w_pre"], h, y, rows, width, scale, eps, kind, code, stream=stream)
        dnb.dnb_op_norm_residual_backward(d["b"], h, d["w_post"], d["gate"], d["w_pre"], d["dh"], d["dy"], db, dr, dwp, dg, dw, rows, width, scale,
                                          eps, kind, code, scratch, stream=stream)
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        d["b"].copy_(torch.randn(rows, width, generator=torch.Generator().manual_seed(turn)).to(torch.bfloat16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
