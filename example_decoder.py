"""The attention half of a decoder block on packed documents, trained for a few steps, then asked for single
tokens over a cache: the sequence operators of the library (attention, rotary positions, the norms around a
block, clipping of all gradients by their norm) in the order in which such a program calls them.  The matrix
products between them are torch's; there is no first norm and no feed-forward half.

    python example_decoder.py [--steps 20] [--width 256] [--heads 8] [--kv-heads 2] [--dtype bf16]

The task: every document is a random sequence of four symbols of its own, and the block has to predict the
next one; which four they are it can only know by attending to what came before.
"""
import argparse
import math

import numpy as np
import torch

import paper_1707_06990_amd as dnb


class Block:
    """Embedding -> attention with rotary positions -> norm, gate and residual -> norm -> symbols.  Parameters
    fp32; activations and the gradients of matrices in `dtype`."""

    def __init__(self, symbols, width, heads, kv_heads, dtype, seed=0):
        self.symbols, self.width, self.heads, self.kv_heads, self.dim = symbols, width, heads, kv_heads, width // heads
        self.dtype, self.code = dtype, dnb.DNB_BF16 if dtype == torch.bfloat16 else dnb.DNB_F32
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda") / math.sqrt(s[-1])  # noqa: E731
        rows = (heads + 2 * kv_heads) * self.dim
        self.p = {"embed": rand(symbols, width) * math.sqrt(width) / 4, "qkv": rand(rows, width), "out": rand(width, width),
                  "head": rand(symbols, width), "w_post": torch.ones(width, device="cuda"), "w_pre": torch.ones(width, device="cuda"),
                  "gate": torch.ones(width, device="cuda")}
        self.turns = (10000.0 ** (-torch.arange(0, self.dim, 2, dtype=torch.float64) / self.dim) / (2 * math.pi)).cuda()
        self.eps, self.scale = 1e-6, 1.0

    def product(self, x, w):
        return x @ w.to(self.dtype).T

    def qkv(self, x, positions, backward=False):
        """Turns the queries and keys of rows that hold queries, keys and values, in place."""
        call = dnb.dnb_op_rope_backward if backward else dnb.dnb_op_rope_forward
        heads = self.heads + self.kv_heads
        call(x, positions, self.turns, x, x.shape[0], heads, self.dim, self.dim, dnb.DNB_ROPE_HALF, 1.0, self.code, x.shape[1], x.shape[1])
        return x.split([self.heads * self.dim, self.kv_heads * self.dim, self.kv_heads * self.dim], 1)

    def norms(self, b, r):
        h, y = torch.empty_like(b), torch.empty_like(b)
        dnb.dnb_op_norm_residual_forward(b, r, self.p["w_post"], self.p["gate"], self.p["w_pre"], h, y, b.shape[0], self.width, self.scale,
                                         self.eps, dnb.DNB_GATE_VECTOR, self.code)
        return h, y


class Step:
    """Plans and workspaces of a training step on documents of the given lengths."""

    def __init__(self, block, lengths):
        m, rows = block, sum(lengths)
        self.m, self.rows = m, rows
        self.offsets = torch.tensor(np.cumsum([0] + list(lengths)), dtype=torch.int32, device="cuda")
        self.positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
        stride = (m.heads + 2 * m.kv_heads) * m.dim
        self.attn = dnb.dnb_attn_create(m.heads, m.kv_heads, m.dim, len(lengths), rows, rows, dtype=m.code, causal=True, q_stride=stride,
                                        k_stride=stride, v_stride=stride)
        scratch = dnb.dnb_op_norm_residual_scratch_bytes(rows, m.width, dnb.DNB_GATE_VECTOR)
        self.workspace = torch.empty(dnb.dnb_attn_workspace_bytes(self.attn), dtype=torch.uint8, device="cuda")
        self.scratch = torch.empty(max(16, scratch), dtype=torch.uint8, device="cuda")
        # the gradients, which are clipped together: matrices in the activations' type, vectors fp32
        self.g = {n: torch.empty(p.shape, dtype=m.dtype if p.dim() == 2 else torch.float32, device="cuda") for n, p in m.p.items()}
        grads = list(self.g.values())
        self.clip = dnb.dnb_clip_create(grads, grads, [dnb.DNB_F32 if g.dtype == torch.float32 else dnb.DNB_BF16 for g in grads])
        self.table = torch.from_numpy(dnb.dnb_clip_table(self.clip)).cuda()
        self.clip_workspace = torch.empty(max(16, dnb.dnb_clip_workspace_bytes(self.clip)), dtype=torch.uint8, device="cuda")
        self.norm = torch.empty(2, device="cuda")

    def gradients(self, tokens, targets, weight):
        """The loss (mean over the rows of weight 1); self.g holds the gradients."""
        m, g = self.m, self.g
        x = m.p["embed"].to(m.dtype)[tokens]
        rows = m.product(x, m.p["qkv"])
        q, k, v = m.qkv(rows, self.positions)
        out = torch.empty(self.rows, m.heads * m.dim, dtype=m.dtype, device="cuda")
        lse = torch.empty(m.heads, self.rows, device="cuda")
        dnb.dnb_attn_forward(self.attn, q, k, v, self.offsets, self.offsets, None, out, lse, self.workspace)
        b = m.product(out, m.p["out"])
        h, y = m.norms(b, x)
        logits = m.product(y, m.p["head"]).float()
        logp = torch.log_softmax(logits, 1)
        count = weight.sum()
        loss = -(logp.gather(1, targets[:, None])[:, 0] * weight).sum() / count

        dlogits = torch.exp(logp)
        dlogits[torch.arange(self.rows, device="cuda"), targets] -= 1
        dlogits = (dlogits * (weight / count)[:, None]).to(m.dtype)
        g["head"].copy_(dlogits.T @ y)
        dy = dlogits @ m.p["head"].to(m.dtype)
        db, dr = torch.empty_like(b), torch.empty_like(b)
        dnb.dnb_op_norm_residual_backward(b, h, m.p["w_post"], m.p["gate"], m.p["w_pre"], torch.zeros_like(h), dy, db, dr, g["w_post"], g["gate"],
                                          g["w_pre"], self.rows, m.width, m.scale, m.eps, dnb.DNB_GATE_VECTOR, m.code, self.scratch)
        g["out"].copy_(db.T @ out)
        dout = db @ m.p["out"].to(m.dtype)
        drows = torch.empty_like(rows)
        dq, dk, dv = drows.split([t.shape[1] for t in (q, k, v)], 1)
        dnb.dnb_attn_backward(self.attn, q, k, v, out, lse, dout, self.offsets, self.offsets, None, dq, dk, dv, self.workspace)
        m.qkv(drows, self.positions, backward=True)
        g["qkv"].copy_(drows.T @ x)
        dx = dr.float() + (drows @ m.p["qkv"].to(m.dtype)).float()
        g["embed"].copy_(torch.zeros_like(m.p["embed"]).index_add_(0, tokens, dx))
        return loss

    def clipped(self, max_norm):
        """Clips self.g; [norm, factor] on the device."""
        dnb.dnb_clip_run(self.clip, self.table, max_norm, self.norm, self.clip_workspace)
        return self.norm

    def close(self):
        dnb.dnb_attn_destroy(self.attn)
        dnb.dnb_clip_destroy(self.clip)


class Cache:
    """Keys and values of `requests` requests with room for `capacity` tokens each; answers one token a request."""

    def __init__(self, block, requests, capacity):
        m = self.m = block
        self.capacity, self.requests, self.used = capacity, requests, 0
        self.k, self.v = (torch.empty(requests * capacity, m.kv_heads * m.dim, dtype=m.dtype, device="cuda") for _ in range(2))
        self.lengths = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.q_offsets = torch.arange(requests + 1, dtype=torch.int32, device="cuda")
        self.k_offsets = self.q_offsets * capacity
        self.attn = dnb.dnb_attn_create(m.heads, m.kv_heads, m.dim, requests, requests, requests * capacity, dtype=m.code, causal=True,
                                        q_stride=(m.heads + 2 * m.kv_heads) * m.dim)
        self.workspace = torch.empty(dnb.dnb_attn_workspace_bytes(self.attn), dtype=torch.uint8, device="cuda")

    def next(self, tokens):
        """Logits after one more token of each request.  ValueError where there is no room for it."""
        if self.used == self.capacity:
            raise ValueError(f"the cache holds {self.capacity} tokens a request")
        self.used += 1
        m = self.m
        x = m.p["embed"].to(m.dtype)[tokens]
        q, k, v = m.qkv(m.product(x, m.p["qkv"]), self.lengths)
        at = (self.k_offsets[:-1] + self.lengths).long()
        self.k[at], self.v[at] = k, v
        self.lengths += 1
        out = torch.empty(self.requests, m.heads * m.dim, dtype=m.dtype, device="cuda")
        lse = torch.empty(m.heads, self.requests, device="cuda")
        dnb.dnb_attn_forward(self.attn, q, self.k, self.v, self.q_offsets, self.k_offsets, self.lengths, out, lse, self.workspace)
        return m.product(m.norms(m.product(out, m.p["out"]), x)[1], m.p["head"]).float()

    def close(self):
        dnb.dnb_attn_destroy(self.attn)


def documents(rng, lengths, symbols):
    """Tokens, the next tokens, and which of those count: those of a document's second half."""
    tokens, targets, weight = [], [], []
    for n in lengths:
        text = rng.choice(symbols, 4, replace=False)[rng.integers(0, 4, n + 1)]
        tokens.append(text[:-1])
        targets.append(text[1:])
        weight.append((np.arange(n) >= n // 2).astype(np.float32))
    put = lambda v, t: torch.tensor(np.concatenate(v), dtype=t, device="cuda")  # noqa: E731
    return put(tokens, torch.long), put(targets, torch.long), put(weight, torch.float32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--symbols", type=int, default=64)
    ap.add_argument("--rate", type=float, default=0.003)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args(argv)
    rng = np.random.default_rng(0)
    block = Block(args.symbols, args.width, args.heads, args.kv_heads, torch.bfloat16 if args.dtype == "bf16" else torch.float32)
    lengths = [250, 127, 64, 33, 500, 1, 90]
    step = Step(block, lengths)
    moments = {n: (torch.zeros_like(p), torch.zeros_like(p)) for n, p in block.p.items()}
    losses = []
    for i in range(args.steps):
        loss = step.gradients(*documents(rng, lengths, args.symbols))
        norm = step.clipped(args.max_norm)
        for n, p in block.p.items():  # Adam
            first, second = moments[n]
            first.lerp_(step.g[n].float(), 0.1)
            second.lerp_(step.g[n].float().square(), 0.01)
            p -= args.rate * (first / (1 - 0.9 ** (i + 1))) / (torch.sqrt(second / (1 - 0.99 ** (i + 1))) + 1e-8)
        losses.append(float(loss))
        if i % 5 == 0 or i + 1 == args.steps:
            print(f"step {i:3d}  loss {losses[-1]:.4f}  gradient norm {float(norm[0]):.4f}", flush=True)
    step.close()
    cache = Cache(block, 4, 40)
    token = torch.tensor(rng.integers(0, args.symbols, 4), device="cuda")
    texts = [token.tolist()]
    for _ in range(20):
        token = cache.next(token).argmax(1)
        texts.append(token.tolist())
    cache.close()
    for r in zip(*texts):  # one request a line
        print(" ".join(map(str, r)), flush=True)
    return losses


if __name__ == "__main__":
    main()
