"""Clipping of the gradients of a CIFAR-shaped training step, where the step leaves them: one after another in one
buffer, clipped in place behind the step on its stream, whole or by the network's parts."""
import math

import pytest
import torch

import workloads as wl
from harness import dev, pack_net

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by_part", [False, True], ids=["whole", "parts"])
def test_gradients_of_a_step(dnb, oracle, by_part):
    cfg = wl.NetCfg(4, 16, 22, 12, 10)
    x, labels, params = wl.make_net_inputs(cfg, affine="random")
    s = oracle.NetShape(cfg.n, cfg.image, cfg.depth, cfg.growth, cfg.classes, cfg.eps)
    flat = pack_net(oracle, s, params)
    _, want, _ = oracle.net_step(s, x, labels, flat)
    net = dnb.dnb_net_create(cfg.n, cfg.image, cfg.depth, cfg.growth, cfg.classes, schedule=dnb.DNB_SCHED_FUSED, eps=cfg.eps)
    p, xd, lab = dev(flat.astype("float32")), dev(x), torch.from_numpy(labels).cuda()
    dp, ws = torch.full_like(p, float("nan")), torch.empty(dnb.dnb_net_workspace_bytes(net), dtype=torch.uint8, device="cuda")
    loss, logits = torch.empty(1, device="cuda"), torch.empty((cfg.n, cfg.classes), device="cuda")
    parts = [dp]
    if by_part:
        spans = [dnb.dnb_net_param_offset(net, i) for i in range(14)]
        assert sum(n for _, n in spans) == p.numel()
        parts = [dp[a:a + n] for a, n in spans]
    plan = dnb.dnb_clip_create(parts, parts, [dnb.DNB_F32] * len(parts))
    table = torch.from_numpy(dnb.dnb_clip_table(plan)).cuda()
    clip_ws, norm = torch.empty(max(16, dnb.dnb_clip_workspace_bytes(plan)), dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
    length = math.sqrt(float((want ** 2).sum()))
    for limit in (0.3 * length, 5 * length):
        dnb.dnb_net_forward(net, xd, lab, p, loss, logits, ws)
        dnb.dnb_net_backward(net, xd, p, dp, ws)
        dnb.dnb_clip_run(plan, table, limit, norm, clip_ws)
        torch.cuda.synchronize()
        coef = min(1.0, limit / (length + 1e-6))
        # the step's own gradients are within 1e-4 of the oracle's
        assert abs(float(norm[0]) - length) <= 1e-4 * length and abs(float(norm[1]) - coef) <= 1e-4 * coef
        assert float((dp.double().cpu() - torch.from_numpy(want) * coef).abs().max()) <= 2e-4 * coef * abs(want).max()
    dnb.dnb_clip_destroy(plan)
    dnb.dnb_net_destroy(net)
