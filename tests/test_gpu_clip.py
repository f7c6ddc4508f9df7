"""Clipping by the global norm against sums in 64 bits, through the C ABI.

Tolerances: squares and at most 64 of their sums in fp32 and sums of those in fp64: the norm is off by at
most (64 + 4) 2^-24 / 2 of itself, the factor by 4 steps more, the result by a product and its rounding."""
import math

import numpy as np
import pytest
import torch

from seq_util import DTYPES, assert_within, half_step

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


def plan_of(dnb, src, dst):
    codes = [dnb.DNB_F32 if t.dtype == torch.float32 else dnb.DNB_BF16 for t in src]
    plan = dnb.dnb_clip_create(src, dst, codes)
    table = torch.from_numpy(dnb.dnb_clip_table(plan)).cuda()
    ws = torch.full((max(16, dnb.dnb_clip_workspace_bytes(plan)),), 255, dtype=torch.uint8, device="cuda")
    return plan, table, ws


SIZES = {"one": [1], "small": [24, 24, 1152, 48, 5184, 1, 7], "borders": [16383, 16384, 16385, 32768, 8, 0, 3], "none": [0, 0],
         "many": [int(x) for x in np.random.default_rng(1).integers(1, 3000, 700)], "large": [3_000_001, 5, 40_000_000]}


@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
@pytest.mark.parametrize("sizes", SIZES, ids=list(SIZES))
@pytest.mark.parametrize("dtype", ["bf16", "f32", "mixed"])
def test_clip(dnb, dtype, sizes, in_place):
    gen = torch.Generator(device="cuda").manual_seed(7)
    kinds = [("bf16", "f32")[i % 2] if dtype == "mixed" else dtype for i in range(len(SIZES[sizes]))]
    raw = [torch.randn(n, generator=gen, device="cuda").mul_(math.exp(i % 3)).to(DTYPES[k]) for i, (n, k) in enumerate(zip(SIZES[sizes], kinds))]
    keep = [t.clone() for t in raw]
    dst = raw if in_place else [torch.full_like(t, float("nan")) for t in raw]
    plan, table, ws = plan_of(dnb, raw, dst)
    norm = torch.full((2,), float("nan"), device="cuda")
    want = math.sqrt(sum(float(t.double().square().sum()) for t in keep))
    for limit in (1e9, 0.25 * want, 0.0):
        for t, k in zip(raw, keep):
            t.copy_(k)
        dnb.dnb_clip_run(plan, table, limit, norm, ws)
        torch.cuda.synchronize()
        n, c = (float(x) for x in norm.cpu())
        coef = min(1.0, limit / (want + 1e-6))
        assert abs(n - want) <= 34 * F * want
        assert abs(c - coef) <= 40 * F * coef
        for t, k in zip(dst, keep):
            if t.numel() > 100000:   # compared on the device
                r = half_step(t.dtype)
                assert bool(((t.double() - k.double() * coef).abs() <= (41 * F + r) * (k.double() * coef).abs()).all())
            else:
                w = k.double().cpu() * coef
                assert_within(t, w, (41 * F + half_step(t.dtype)) * w.abs(), "clipped")
    dnb.dnb_clip_destroy(plan)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tensors_off_16_bytes(dnb, dtype):
    base = torch.randn(50_000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DTYPES[dtype])
    out = torch.zeros_like(base)
    cut = [(1, 20_000), (20_003, 20_004), (20_005, 50_000)]
    plan, table, ws = plan_of(dnb, [base[a:b] for a, b in cut], [out[a:b] for a, b in cut])
    norm = torch.empty(2, device="cuda")
    dnb.dnb_clip_run(plan, table, 1.0, norm, ws)
    mine = torch.zeros(50_000, dtype=torch.bool)
    for a, b in cut:
        mine[a:b] = True
    want = base.double().cpu() * mine
    coef = 1.0 / (float(want.square().sum().sqrt()) + 1e-6)
    assert_within(out, want * coef, (41 * F + half_step(base.dtype)) * (want * coef).abs(), "clipped")
    dnb.dnb_clip_destroy(plan)


def test_values_that_are_not_finite(dnb):
    """An infinite gradient makes the factor 0 (and itself NaN), a NaN makes everything NaN, as the formula does."""
    for bad in (float("inf"), float("nan")):
        g = [torch.ones(1000, device="cuda"), torch.ones(77, device="cuda")]
        g[1][5] = bad
        dst = [torch.zeros_like(t) for t in g]
        plan, table, ws = plan_of(dnb, g, dst)
        norm = torch.empty(2, device="cuda")
        dnb.dnb_clip_run(plan, table, 1.0, norm, ws)
        coef = torch.clamp(1.0 / (torch.cat(g).square().sum().sqrt() + 1e-6), max=1.0)
        for a, b in zip(dst, g):
            assert torch.equal(torch.nan_to_num(a, nan=-7.0), torch.nan_to_num(b * coef, nan=-7.0))
        dnb.dnb_clip_destroy(plan)


def test_repeats_bit_for_bit_and_in_a_graph(dnb):
    g = [torch.empty(n, device="cuda", dtype=torch.bfloat16) for n in (100_000, 3, 70_001)]
    dst = [torch.empty_like(t) for t in g]
    plan, table, ws = plan_of(dnb, g, dst)
    norm = torch.empty(2, device="cuda")
    dnb.dnb_clip_run(plan, table, 1.0, norm, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dnb.dnb_clip_run(plan, table, 1.0, norm, ws)
    for turn in range(3):
        for t in g:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(turn)).to(t.dtype))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*dst, norm)]
        dnb.dnb_clip_run(plan, table, 1.0, norm, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*dst, norm)))
    dnb.dnb_clip_destroy(plan)
