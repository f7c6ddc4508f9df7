"""Clipping of gradients whose squares, or whose norm, fp32 does not hold, against sums in 64 bits.

Tolerances: the norm is rounded to fp32 once (sums in 64 bits), the factor once from a quotient in 64 bits,
a result is a product (one rounding; another where the factor is applied in two) and its rounding to its
type.  A factor below fp32's normal range is off by half of its last place, 2^-150."""
import math

import pytest
import torch

from seq_util import DTYPES, assert_within, half_step

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


# magnitude of the values, limit of the norm
RANGES = {"exploding": (1e20, 1.0), "largest": (3e38, 1.0), "largest_over_a_large_limit": (3e38, 1e30), "mixed": (None, 0.5),
          "vanishing": (1e-30, 1.0), "vanishing_over_a_small_limit": (1e-30, 1e-37), "squares_at_the_border": (2e-20, 1e-3)}


@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
@pytest.mark.parametrize("name", RANGES, ids=list(RANGES))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_any_finite_magnitude(dnb, dtype, name, in_place):
    size, limit = RANGES[name]
    gen = torch.Generator().manual_seed(3)
    counts = [1, 77, 16385, 40000, 8]
    raw = []
    for i, n in enumerate(counts):
        level = size if size else (1e25, 1e-25, 1.0, 1e-3, 1e19)[i]
        v = (torch.rand(n, generator=gen) * 0.5 + 0.5) * torch.where(torch.rand(n, generator=gen) < 0.5, -1.0, 1.0)
        raw.append((v * level).to(DTYPES[dtype]))
    assert all(bool(torch.isfinite(t.float()).all()) for t in raw)
    norm_want = math.sqrt(sum(float(t.double().square().sum()) for t in raw))
    coef = min(1.0, limit / (norm_want + 1e-6))
    src = [t.cuda() for t in raw]
    dst = src if in_place else [torch.full_like(t, float("nan")) for t in src]
    plan = dnb.dnb_clip_create(src, dst, [dnb.DNB_BF16 if dtype == "bf16" else dnb.DNB_F32] * len(src))
    table = torch.from_numpy(dnb.dnb_clip_table(plan)).cuda()
    ws = torch.full((max(16, dnb.dnb_clip_workspace_bytes(plan)),), 255, dtype=torch.uint8, device="cuda")
    norm = torch.full((2,), float("nan"), device="cuda")
    dnb.dnb_clip_run(plan, table, limit, norm, ws)
    torch.cuda.synchronize()
    got_norm, got_coef = (float(x) for x in norm.cpu())
    if norm_want * (1 - 2 * F) > torch.finfo(torch.float32).max:   # the norm itself is beyond fp32; the factor is not
        assert got_norm == math.inf
    else:
        assert abs(got_norm - norm_want) <= 1.01 * F * norm_want + 2.0 ** -150
    # max_norm is an fp32 argument: rounded once
    assert abs(got_coef - coef) <= 2.02 * F * coef + 2.0 ** -150
    for t, k in zip(dst, raw):
        w = k.double() * coef
        # below the normal range one rounding is half of the last place there
        least = 2.0 ** -150 if dtype == "f32" else 2.0 ** -134
        assert_within(t, w, (5 * F + half_step(t.dtype)) * w.abs() + 2 * least, "clipped")
    dnb.dnb_clip_destroy(plan)
