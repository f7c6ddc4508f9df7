"""Definitions of the sequence operators in 64 bits, on the CPU, with bounds on what rounding may add."""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(dtype):
    """Largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def visible(nq, nk, causal):
    if not causal:
        return torch.ones(nq, nk, dtype=torch.bool)
    return torch.arange(nk)[None, :] <= torch.arange(nq)[:, None] + nk - nq


def attn_pieces(q_offsets, k_offsets, k_lengths):
    for s in range(len(q_offsets) - 1):
        q = slice(q_offsets[s], q_offsets[s + 1])
        n = k_offsets[s + 1] - k_offsets[s] if k_lengths is None else k_lengths[s]
        yield q, slice(k_offsets[s], k_offsets[s] + n)


def attn_forward(q, k, v, q_offsets, k_offsets, k_lengths, causal, scale=None):
    """(out, lse, bound of out's rounding, bound of lse's) for tensors of any type, computed in 64 bits.

    The type is where q is kept: the probabilities are rounded to it for the second product, and the
    result once.  fp32 sums of n terms are off by at most n steps of 2^-24 of the sum of magnitudes; a
    score that is off by e changes its probability by a factor 1 + e."""
    r, f = half_step(q.dtype), 2.0 ** -24
    r_p = r if q.dtype != torch.float32 else 0.0
    q, k, v = q.double(), k.double(), v.double()
    heads, per, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = scale or 1 / math.sqrt(d)
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((heads, q.shape[0]), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    for qs, ks in attn_pieces(q_offsets, k_offsets, k_lengths):
        seen = visible(qs.stop - qs.start, ks.stop - ks.start, causal)
        if seen.numel() == 0:
            continue
        for h in range(heads):
            a, b, c = q[qs, h], k[ks, h // per], v[ks, h // per]
            s = (a @ b.T * scale).masked_fill(~seen, -math.inf)
            lse[h, qs] = torch.logsumexp(s, 1)
            p = torch.nan_to_num(torch.softmax(s, 1), nan=0.0)
            out[qs, h] = p @ c
            size = (a.abs() @ b.abs().T * scale).masked_fill(~seen, 0).amax(1, keepdim=True)
            e = f * ((d + 8) * size + seen.shape[1] + 16)
            tol[qs, h] = (r_p + 2 * e) * (p @ c.abs()) + r * out[qs, h].abs()
            lse_tol[h, qs] = (2 * e)[:, 0] + 4 * f * torch.nan_to_num(lse[h, qs], neginf=0).abs()
    return out, lse, tol, lse_tol


def attn_backward(q, k, v, out, lse, dout, q_offsets, k_offsets, k_lengths, causal, scale=None):
    """(dq, dk, dv) and the bounds of their rounding, from the given out and lse."""
    r, f = half_step(q.dtype), 2.0 ** -24
    r_p = r if q.dtype != torch.float32 else 0.0
    q, k, v, out, lse, dout = (t.double() for t in (q, k, v, out, lse, dout))
    heads, per, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = scale or 1 / math.sqrt(d)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    tq, tk, tv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for qs, ks in attn_pieces(q_offsets, k_offsets, k_lengths):
        seen = visible(qs.stop - qs.start, ks.stop - ks.start, causal)
        if seen.numel() == 0:
            continue
        n = max(seen.shape[0] * per, seen.shape[1])
        for h in range(heads):
            g = h // per
            a, b, c, o, do = q[qs, h], k[ks, g], v[ks, g], out[qs, h], dout[qs, h]
            p = torch.exp((a @ b.T * scale).masked_fill(~seen, -math.inf) - lse[h, qs][:, None])
            p = torch.nan_to_num(p, nan=0.0)   # rows that see nothing: exp(-inf + inf)
            dp, big = do @ c.T, do.abs() @ c.abs().T
            D, bigD = (do * o).sum(1, keepdim=True), (do * o).abs().sum(1, keepdim=True)
            ds = p * (dp - D)
            size = (a.abs() @ b.abs().T * scale).masked_fill(~seen, 0).amax(1, keepdim=True)
            e = f * ((d + 8) * size + 4 * torch.nan_to_num(lse[h, qs][:, None], neginf=0).abs() + 16)
            ep = (r_p + e + f * n) * p
            es = (r_p + e + f * n) * ds.abs() + p * f * (d + 4) * (big + bigD)
            # bf16: sum_d dout out of rows that see few keys may be taken from p and dout v^T instead; the given out
            # is off by its rounding, half a step, and so is the sum from it
            few = seen.sum(1, keepdim=True) <= 160
            es = es + few * r_p * p * (do.abs() * o.abs()).sum(1, keepdim=True)
            dq[qs, h] = scale * ds @ b
            tq[qs, h] = scale * es @ b.abs()
            dk[ks, g] += scale * ds.T @ a
            tk[ks, g] += scale * es.T @ a.abs()
            dv[ks, g] += p.T @ do
            tv[ks, g] += ep.T @ do.abs()
    return (dq, dk, dv), (tq + r * dq.abs(), tk + r * dk.abs(), tv + r * dv.abs())


def assert_within(got, want, tol, what):
    got = got.detach().double().cpu()
    bad = ~((got - want).abs() <= tol) & ~(got == want)
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i].item()} for {want[i].item()} "
                             f"(allowed {tol[i].item()})")
