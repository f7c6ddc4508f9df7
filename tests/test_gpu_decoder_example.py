"""The example's training step and its single-token form (example_decoder.py) against the same block in 64
bits with gradients by automatic differentiation, and against each other.

fp32: every product and every operator adds some steps of 2^-24 of sums of up to a few hundred terms of
order one, over some ten operations: 1e-4 of a gradient's largest value is far above that and far below any
mistake."""
import math

import numpy as np
import pytest
import torch

import example_decoder as ex

pytestmark = pytest.mark.gpu


def plain(block, tokens, targets, weight, lengths):
    """Loss and gradients in 64 bits on the CPU."""
    m = block
    p = {n: t.double().cpu().requires_grad_() for n, t in m.p.items()}
    tokens, targets, weight = tokens.cpu(), targets.cpu(), weight.double().cpu()
    x = p["embed"][tokens]
    q, k, v = (x @ p["qkv"].T).split([m.heads * m.dim, m.kv_heads * m.dim, m.kv_heads * m.dim], 1)
    pos = torch.cat([torch.arange(n) for n in lengths]).double()
    angle = 2 * math.pi * pos[:, None] * m.turns.cpu()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def turn(t):
        a, b = t.reshape(t.shape[0], -1, m.dim).chunk(2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2)
    q, k, v = turn(q), turn(k), v.reshape(v.shape[0], -1, m.dim)
    out, at = [], 0
    for n in lengths:
        s = slice(at, at + n)
        at += n
        mask = torch.ones(n, n, dtype=torch.bool).triu(1)
        rows = []
        for h in range(m.heads):
            g = h * m.kv_heads // m.heads
            score = (q[s, h] @ k[s, g].T / math.sqrt(m.dim)).masked_fill(mask, -math.inf)
            rows.append(torch.softmax(score, 1) @ v[s, g])
        out.append(torch.cat(rows, 1))
    b = torch.cat(out) @ p["out"].T
    unit = lambda t: t / torch.sqrt(t.square().mean(1, keepdim=True) + m.eps)
    h = m.scale * x + p["gate"] * (unit(b) * p["w_post"])
    logits = (unit(h) * p["w_pre"]) @ p["head"].T
    loss = -(torch.log_softmax(logits, 1).gather(1, targets[:, None])[:, 0] * weight).sum() / weight.sum()
    loss.backward()
    return float(loss.detach()), {n: t.grad for n, t in p.items()}, logits.detach()


LENGTHS = [70, 33, 1, 128]


def test_a_training_step(dnb):
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=1)
    step = ex.Step(block, LENGTHS)
    data = ex.documents(np.random.default_rng(2), LENGTHS, 40)
    loss = float(step.gradients(*data))
    want, grads, _ = plain(block, *data, LENGTHS)
    assert abs(loss - want) <= 1e-5 * abs(want)
    for n, g in grads.items():
        assert float((step.g[n].double().cpu() - g).abs().max()) <= 1e-4 * float(g.abs().max()), n
    norm = math.sqrt(sum(float(g.square().sum()) for g in grads.values()))
    got = step.clipped(0.5 * norm).cpu()
    assert abs(float(got[0]) - norm) <= 1e-4 * norm and abs(float(got[1]) - 0.5) <= 1e-4
    for n, g in grads.items():
        assert float((step.g[n].double().cpu() - 0.5 * g).abs().max()) <= 1e-4 * float(g.abs().max()), n
    step.close()


def test_single_tokens_give_the_logits_of_the_whole_document(dnb):
    """Token by token over a cache, the logits of a document are those of one pass over it."""
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=3)
    lengths = [50, 50]
    data = ex.documents(np.random.default_rng(4), lengths, 40)
    _, _, logits = plain(block, *data, lengths)
    cache = ex.Cache(block, 2, 64)
    text = data[0].reshape(2, 50)
    for i in range(50):
        got = cache.next(text[:, i]).double().cpu()
        assert float((got - logits.reshape(2, 50, -1)[:, i]).abs().max()) <= 1e-4 * float(logits.abs().max()), i
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_command_learns(dnb, dtype):
    losses = ex.main(["--steps", "60", "--dtype", dtype])
    assert all(math.isfinite(x) for x in losses)
    assert losses[-1] < 0.9 * losses[0], losses
