"""Performance cases of the sequence operators: attention over packed sequences, rotary positions,
the norms around a block with its gate and residual scale, and the clipping of many gradients by
their global norm.

A case is a dict of plain values.  "kind" is attn, rope, norm or clip; "direction" is forward,
backward or step (forward, then backward with what the forward left).  Lengths of packed sequences
are texts of whole numbers with commas between them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _attn(name, dtype, q_lengths, k_lengths, heads, kv_heads, head_dim, causal=True, direction="forward", capacity=0):
    """capacity: 0 for packed keys, else the rows that every sequence has in a cache, of which its length is in use."""
    return {"name": name, "kind": "attn", "dtype": dtype, "direction": direction, "q_lengths": ",".join(map(str, q_lengths)),
            "k_lengths": ",".join(map(str, k_lengths)), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "causal": causal, "capacity": capacity}


def _rope(name, dtype, rows, heads, head_dim, rotary_dim, interleaved, scaling, far, direction="forward"):
    return {"name": name, "kind": "rope", "dtype": dtype, "direction": direction, "rows": rows, "heads": heads,
            "head_dim": head_dim, "rotary_dim": rotary_dim, "interleaved": interleaved, "scaling": scaling, "far": far}


def _norm(name, dtype, rows, width, gate, post, scale, direction):
    return {"name": name, "kind": "norm", "dtype": dtype, "direction": direction, "rows": rows, "width": width,
            "gate": gate, "post": post, "scale": scale}


def _clip(name, dtype, model, depth, width, growth, max_norm):
    return {"name": name, "kind": "clip", "dtype": dtype, "direction": "forward", "model": model, "depth": depth,
            "width": width, "growth": growth, "max_norm": max_norm}


def listed():
    tokens = [1] * 16
    held = [8192, 6001, 5120, 4097, 4096, 3500, 2777, 2048, 1999, 1024, 700, 513, 128, 64, 17, 1]
    packed, ragged = [2048, 2048, 1333, 1024, 515, 200, 64, 1], [4096, 3333, 2900, 1531, 640, 97]
    return [
        # answering: one new token for each of sixteen requests, over caches that are filled unevenly
        _attn("attn_token", "bf16", tokens, held, 32, 8, 128, capacity=8192),
        # the prompts of a batch of requests, packed, before the first token is answered
        _attn("attn_prompt", "bf16", ragged, ragged, 32, 8, 128),
        # a training step on packed documents
        _attn("attn_train", "bf16", packed, packed, 16, 4, 128, direction="step"),
        # every pixel of a 14x14 feature map looks at every other: a training step in fp32, 32 images
        _attn("attn_pixels", "f32", [196] * 32, [196] * 32, 8, 8, 64, causal=False, direction="step"),
        # the smallest step: launches and latency
        _attn("attn_short", "bf16", [33], [33], 8, 2, 64, direction="step"),
        # queries and keys of one new token a request, at far positions of a stretched context
        _rope("rope_token", "bf16", 16, 40, 128, 128, False, "yarn", 131072),
        # queries and keys of a training step, half of each head turned, pairs side by side
        _rope("rope_train", "f32", 8191, 24, 128, 64, True, "none", 8191, "step"),
        # the norms around a block for one new token a request
        _norm("norm_token", "bf16", 16, 4096, "vector", True, 1.0, "forward"),
        # ... and of a training step's backward pass on a long packed batch
        _norm("norm_backward", "bf16", 16381, 4096, "vector", True, 0.5, "backward"),
        # a training step in fp32 at the width of the ImageNet-shaped network's last features, gated by value
        _norm("norm_step", "f32", 6272, 2208, "full", True, 0.7071, "step"),
        # the gradients of the CIFAR-shaped training step, tensor by tensor: some hundred small tensors
        _clip("clip_small", "f32", "dense", 100, 24, 12, 1.0),
        # the gradients of a decoder of 12 layers, bf16
        _clip("clip_large", "bf16", "decoder", 12, 2048, 0, 1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = (max(most.get(c["kind"], (0, 0))[0], w["flops"]), max(most.get(c["kind"], (0, 0))[1], w["bytes"]))
    kind = rng.choice(["attn", "attn", "attn", "rope", "norm", "clip"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        direction = rng.choice(["forward", "step"])
        if kind == "attn":
            kv = rng.choice([1, 2, 3, 4, 8])
            heads = kv * rng.choice([1, 1, 2, 3, 4, 7, 8])
            dim = rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
            form = rng.choice(["token", "prompt", "prompt", "chunk"])
            n = _log_int(rng, 1, 48 if form == "token" else 12)
            ks = [_log_int(rng, 1, 8192 if form == "token" else 4096) for _ in range(n)]
            if form == "token":
                c = _attn("", dtype, [1] * n, ks, heads, kv, dim, capacity=max(ks) + rng.randint(0, 99))
            elif form == "chunk":  # the last part of a prompt over all keys so far; some with more queries than keys
                c = _attn("", dtype, [_log_int(rng, 1, k + 3) for k in ks], ks, heads, kv, dim, direction=direction)
            else:
                c = _attn("", dtype, ks, ks, heads, kv, dim, rng.random() < 0.7, direction)
        elif kind == "rope":
            dim = rng.choice([32, 64, 80, 128])
            rows = _log_int(rng, 1, 8191)
            c = _rope("", dtype, rows, rng.randint(1, 40), dim, rng.choice([dim, dim, dim // 2]), rng.random() < 0.5,
                      rng.choice(["none", "linear", "ntk", "yarn"]), _log_int(rng, 64, 131072), direction)
        elif kind == "norm":
            if dtype == "bf16":
                direction = rng.choice(["forward", "backward"])
            c = _norm("", dtype, _log_int(rng, 1, 16381), 8 * _log_int(rng, 8, 1024), rng.choice(["none", "vector", "full"]),
                      rng.random() < 0.7, rng.choice([1.0, 0.5, 0.7071]), direction)
        else:
            if rng.random() < 0.5:
                c = _clip("", dtype, "dense", 6 * rng.randint(4, 41) + 4, 2 * rng.choice([12, 16, 24]), rng.choice([12, 16, 24]),
                          rng.choice([0.25, 1.0, 5.0]))
            else:
                c = _clip("", dtype, "decoder", rng.randint(1, 12), 8 * _log_int(rng, 16, 256), 0, rng.choice([0.25, 1.0, 5.0]))
        w = work(c)
        padded = 1
        if kind == "attn":
            q, k = _lengths(c)
            padded = len(q) * max(q) * max(k) * c["heads"] / (6 * 4096 * 4096 * 32)
        # fp32 products of matrices are a sixteenth as fast
        if w["flops"] * (16 if dtype == "f32" and kind == "attn" else 1) <= most[kind][0] and w["bytes"] <= most[kind][1] and padded <= 1:
            del c["name"]
            return c


# ---------------------------------------------------------------- sizes

def _lengths(case):
    return [int(v) for v in case["q_lengths"].split(",")], [int(v) for v in case["k_lengths"].split(",")]


def _pairs(nq, nk, causal):
    """How many (query, key) pairs see each other; query i of nq sees keys up to i + nk - nq."""
    if not causal:
        return nq * nk
    first = max(0, nq - nk)  # queries before this one see nothing
    n = nq - first
    return n * (nk - nq + first + 1) + n * (n - 1) // 2


def _sizes(case):
    """Values of each gradient tensor: of a DenseNet-BC of `depth` layers (`width` channels after the
    first convolution), or of a decoder of `depth` blocks."""
    w, out = case["width"], []
    if case["model"] == "decoder":
        for _ in range(case["depth"]):
            out += [w, w * w, w * w // 4, w * w // 4, w * w, w, 3 * w * w, 3 * w * w, 3 * w * w, w, w]
        return out + [w, 16000 * w]
    k, c = case["growth"], w
    out.append(27 * w)
    for block in range(3):
        for _ in range((case["depth"] - 4) // 6):
            out += [c, c, 4 * k * c, 4 * k, 4 * k, 36 * k * k]
            c += k
        if block < 2:
            out += [c, c, c * (c // 2)]
            c //= 2
    return out + [c, c, 10 * c, 10]


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    step, back = case["direction"] == "step", case["direction"] == "backward"
    if case["kind"] == "attn":
        q, k = _lengths(case)
        nq, nk, d = sum(q), sum(k), case["head_dim"]
        pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(q, k)) * case["heads"]
        # q, k, v read, out and the rows' log sums written; for the gradients out, its gradient, q, k, v, and three written
        byt = (2 * nq * case["heads"] + 2 * nk * case["kv_heads"]) * d * size + 4 * nq * case["heads"]
        if step:
            byt += (4 * nq * case["heads"] + 4 * nk * case["kv_heads"]) * d * size + 4 * nq * case["heads"]
        return {"bytes": byt, "flops": (14 if step else 4) * d * pairs}
    if case["kind"] == "rope":
        n = case["rows"] * case["heads"] * case["head_dim"]
        return {"bytes": (2 if step else 1) * (2 * n * size + 4 * case["rows"]), "flops": (2 if step else 1) * 3 * n}
    if case["kind"] == "norm":
        n, full = case["rows"] * case["width"], case["gate"] == "full"
        fwd, bwd = (4 + full) * n * size, (6 + 2 * full) * n * size
        return {"bytes": bwd if back else fwd + bwd if step else fwd, "flops": n * (24 if back else 34 if step else 10)}
    n = sum(_sizes(case))
    return {"bytes": 2 * n * size, "flops": 3 * n}


# ---------------------------------------------------------------- inputs

def _rand(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _frequencies(case):
    """Turning angle per position of each pair, in double precision, and the factor on the turned values
    (base 10000; stretched contexts: four times the trained 4096 positions)."""
    dim, base, factor, trained = case["rotary_dim"], 10000.0, 4.0, 4096
    if case["scaling"] == "ntk":
        base *= factor ** (dim / (dim - 2))
    f = base ** (-np.arange(0, dim, 2, dtype=np.float64) / dim)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] != "yarn":
        return f, 1.0
    turns = trained * f / (2 * math.pi)  # full turns over the trained context: over 32 kept, under 1 stretched
    keep = np.clip((turns - 1) / (32 - 1), 0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "attn":
        q, k = _lengths(case)
        h, g, d, cap = case["heads"], case["kv_heads"], case["head_dim"], case["capacity"]
        nk = cap * len(k) if cap else sum(k)
        s["q"], s["k"], s["v"] = (_rand(gen, (n, m, d), dt) for n, m in ((sum(q), h), (nk, g), (nk, g)))
        s["dout"] = _rand(gen, (sum(q), h, d), dt)
        ints = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
        s["q_offsets"] = ints(np.cumsum([0] + q))
        s["k_offsets"] = ints(np.arange(len(k) + 1) * cap if cap else np.cumsum([0] + k))
        s["k_lengths"] = ints(k) if cap else None
        s["max_q"], s["max_k"] = max(q), max(k)
    elif case["kind"] == "rope":
        shape = (case["rows"], case["heads"], case["head_dim"])
        s["x"], s["dy"] = _rand(gen, shape, dt), _rand(gen, shape, dt)
        s["positions"] = torch.randint(0, case["far"], (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        f, s["factor"] = _frequencies(case)
        s["frequencies"] = torch.tensor(f, device="cuda")
    elif case["kind"] == "norm":
        shape, w = (case["rows"], case["width"]), case["width"]
        for name in ("b", "r", "dh", "dy"):
            s[name] = _rand(gen, shape, dt)
        s["h"] = _rand(gen, shape, dt, 1.5)
        s["w_post"] = 1 + _rand(gen, (w,), torch.float32, 0.2) if case["post"] else None
        s["w_pre"] = 1 + _rand(gen, (w,), torch.float32, 0.2)
        s["gate"] = {"none": None, "vector": _rand(gen, (w,), torch.float32, 0.5), "full": None}[case["gate"]]
        if case["gate"] == "full":
            s["gate"] = torch.sigmoid(_rand(gen, shape, torch.float32)).to(dt)
        s["eps"] = 1e-6
    else:
        sizes = _sizes(case)
        # every tensor starts on a multiple of 64 values of one arena, as a trainer lays its gradients out
        starts = np.concatenate([[0], np.cumsum([-(-n // 64) * 64 for n in sizes])])
        s["sizes"], s["starts"] = sizes, [int(v) for v in starts]
        level = torch.exp(torch.randn(len(sizes), generator=gen, device="cuda") - 5)
        s["raw"] = torch.zeros(int(starts[-1]), dtype=dt, device="cuda")
        for i, (a, n) in enumerate(zip(s["starts"], sizes)):
            s["raw"][a:a + n] = _rand(gen, (n,), dt, level[i])
        s["clipped"] = torch.zeros_like(s["raw"])
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """Plans and workspaces, which a user's program makes once and keeps."""
    import paper_1707_06990_amd as dnb
    c = s["case"]
    dt = dnb.DNB_F32 if c["dtype"] == "f32" else dnb.DNB_BF16
    nbytes = lambda n: torch.empty(max(16, n), dtype=torch.uint8, device="cuda")  # noqa: E731
    s["dnb"], s["dtype"] = dnb, dt
    if c["kind"] == "attn":
        q, k = s["q"], s["k"]
        s["plan"] = dnb.dnb_attn_create(c["heads"], c["kv_heads"], c["head_dim"], s["q_offsets"].numel() - 1, q.shape[0],
                                        k.shape[0], dtype=dt, causal=c["causal"])
        s["workspace"] = nbytes(dnb.dnb_attn_workspace_bytes(s["plan"]))
        s["out"], s["lse"] = torch.empty_like(q), torch.empty((c["heads"], q.shape[0]), device="cuda")
        s["dq"], s["dk"], s["dv"] = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    elif c["kind"] == "rope":
        s["turns"] = s["frequencies"] / (2 * math.pi)
        s["y"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    elif c["kind"] == "norm":
        s["scratch"] = nbytes(dnb.dnb_op_norm_residual_scratch_bytes(c["rows"], c["width"], _gate_kind(s)))
        for name, like in (("h_new", "b"), ("y", "b"), ("db", "b"), ("dr", "b"), ("dw_pre", "w_pre"), ("dw_post", "w_post"), ("dgate", "gate")):
            s[name] = None if s[like] is None else torch.empty_like(s[like])
    else:
        views = lambda t: [t[a:a + n] for a, n in zip(s["starts"], s["sizes"])]  # noqa: E731
        s["plan"] = dnb.dnb_clip_create(views(s["raw"]), views(s["clipped"]), [dt] * len(s["sizes"]))
        s["table"] = torch.from_numpy(dnb.dnb_clip_table(s["plan"])).cuda()
        s["workspace"] = nbytes(dnb.dnb_clip_workspace_bytes(s["plan"]))
        s["norm"] = torch.empty(2, device="cuda")


def _gate_kind(s):
    dnb = s["dnb"]
    return {"none": dnb.DNB_GATE_NONE, "vector": dnb.DNB_GATE_VECTOR, "full": dnb.DNB_GATE_FULL}[s["case"]["gate"]]


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    dnb, c = s["dnb"], s["case"]
    step, back = c["direction"] == "step", c["direction"] == "backward"
    if c["kind"] == "attn":
        dnb.dnb_attn_forward(s["plan"], s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s["k_lengths"], s["out"], s["lse"],
                             s["workspace"])
        if not step:
            return s["out"], s["lse"]
        dnb.dnb_attn_backward(s["plan"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["q_offsets"], s["k_offsets"],
                              s["k_lengths"], s["dq"], s["dk"], s["dv"], s["workspace"])
        return s["out"], s["lse"], s["dq"], s["dk"], s["dv"]
    if c["kind"] == "rope":
        order = dnb.DNB_ROPE_INTERLEAVED if c["interleaved"] else dnb.DNB_ROPE_HALF
        size = (c["rows"], c["heads"], c["head_dim"], c["rotary_dim"])
        dnb.dnb_op_rope_forward(s["x"], s["positions"], s["turns"], s["y"], *size, order, s["factor"], s["dtype"])
        if not step:
            return s["y"]
        dnb.dnb_op_rope_backward(s["dy"], s["positions"], s["turns"], s["dx"], *size, order, s["factor"], s["dtype"])
        return s["y"], s["dx"]
    if c["kind"] == "norm":
        if not back:
            dnb.dnb_op_norm_residual_forward(s["b"], s["r"], s["w_post"], s["gate"], s["w_pre"], s["h_new"], s["y"], c["rows"],
                                             c["width"], c["scale"], s["eps"], _gate_kind(s), s["dtype"])
        if not (step or back):
            return s["h_new"], s["y"]
        dnb.dnb_op_norm_residual_backward(s["b"], s["h"] if back else s["h_new"], s["w_post"], s["gate"], s["w_pre"], s["dh"], s["dy"],
                                          s["db"], s["dr"], s["dw_post"], s["dgate"], s["dw_pre"], c["rows"], c["width"], c["scale"],
                                          s["eps"], _gate_kind(s), s["dtype"], s["scratch"])
        grads = [s[n] for n in ("db", "dr", "dw_pre", "dw_post", "dgate") if s[n] is not None]
        return grads if back else [s["h_new"], s["y"]] + grads
    dnb.dnb_clip_run(s["plan"], s["table"], c["max_norm"], s["norm"], s["workspace"])
    return s["clipped"], s["norm"]


# ---------------------------------------------------------------- the plain forms

def _padded(offsets, lengths, longest):
    """Rows of every sequence side by side (sequences, longest), those past its end on its first row, and which are its own."""
    at = torch.arange(longest, device="cuda")
    real = at[None, :] < lengths[:, None]
    return offsets[:-1, None].long() + at[None, :] * real, real


def _plain_attn(s):
    c = s["case"]
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    per, dt, scale = h // g, s["q"].dtype, 1 / math.sqrt(d)
    qo, ko = s["q_offsets"], s["k_offsets"]
    ql = qo[1:] - qo[:-1]
    kl = ko[1:] - ko[:-1] if s["k_lengths"] is None else s["k_lengths"]
    rows_q, real_q = _padded(qo, ql, s["max_q"])
    rows_k, real_k = _padded(ko, kl, s["max_k"])
    n, mq, mk = rows_q.shape[0], s["max_q"], s["max_k"]
    heads_first = lambda t, r: t[r].float().transpose(1, 2)  # noqa: E731  (sequences, heads, rows, head_dim)
    by_query = lambda t: heads_first(t, rows_q).reshape(n, g, per * mq, d)  # noqa: E731
    q, k, v = by_query(s["q"]), heads_first(s["k"], rows_k).contiguous(), heads_first(s["v"], rows_k).contiguous()
    seen = real_q[:, :, None] & real_k[:, None, :]
    if c["causal"]:
        last = torch.arange(mq, device="cuda")[None, :] + (kl - ql)[:, None]
        seen &= torch.arange(mk, device="cuda")[None, None, :] <= last[:, :, None]
    seen = seen[:, None, None].expand(n, g, per, mq, mk).reshape(n, g, per * mq, mk) if per > 1 else seen[:, None]
    p = (q @ k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(p.sub_(top))
    total = p.sum(3, keepdim=True)
    lse = torch.log(total) + top
    p /= torch.where(total == 0, torch.ones_like(total), total)
    row_seq = torch.repeat_interleave(torch.arange(n, device="cuda"), ql, output_size=s["q"].shape[0])
    row_at = torch.arange(s["q"].shape[0], device="cuda") - qo.long()[row_seq]
    back_q = lambda t: t.reshape(n, h, mq, -1).transpose(1, 2)[row_seq, row_at].to(dt)  # noqa: E731
    out = back_q(p @ v)
    lse = lse.reshape(n, h, mq).transpose(1, 2)[row_seq, row_at].transpose(0, 1).contiguous()
    if c["direction"] != "step":
        return out, lse
    do = by_query(s["dout"]) * real_q[:, None, None].expand(n, g, per, mq).reshape(n, g, per * mq, 1)
    dv = p.transpose(2, 3).contiguous() @ do
    ds = do @ v.transpose(2, 3).contiguous()
    ds = p * ds.sub_((p * ds).sum(3, keepdim=True)) * scale
    dq = back_q(ds @ k)
    dk = ds.transpose(2, 3).contiguous() @ q
    key_seq = torch.repeat_interleave(torch.arange(n, device="cuda"), kl, output_size=s["k"].shape[0])
    key_at = torch.arange(s["k"].shape[0], device="cuda") - ko.long()[key_seq]
    back_k = lambda t: t.transpose(1, 2)[key_seq, key_at].to(dt)  # noqa: E731
    return out, lse, dq, back_k(dk), back_k(dv)


def _plain_turn(x, s, sign):
    c = s["case"]
    dim, half = c["rotary_dim"], c["rotary_dim"] // 2
    angle = s["positions"].double()[:, None] * s["frequencies"][None, :]  # far positions need more than 32 bits
    cos, sin = (torch.cos(angle) * s["factor"]).float()[:, None], (sign * torch.sin(angle) * s["factor"]).float()[:, None]
    y = x.float()
    turned = y[..., :dim]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if c["interleaved"] else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).reshape(turned.shape) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., dim:]), -1).to(x.dtype)


def _plain_norm(s):
    c = s["case"]
    dt, eps = s["b"].dtype, s["eps"]
    step, back = c["direction"] == "step", c["direction"] == "backward"
    b = s["b"].float()
    inv_b = torch.rsqrt((b * b).mean(1, keepdim=True) + eps) if c["post"] else 1.0
    xb = b * inv_b
    wp = s["w_post"] if c["post"] else 1.0
    gate = s["gate"].float() if s["gate"] is not None else 1.0
    got = []
    if back:
        h = s["h"].float()
    else:
        h = c["scale"] * s["r"].float() + gate * (xb * wp)
    inv_h = torch.rsqrt((h * h).mean(1, keepdim=True) + eps)
    xh = h * inv_h
    if not back:
        got = [h.to(dt), (xh * s["w_pre"]).to(dt)]
    if not (step or back):
        return got
    dy = s["dy"].float()
    t = dy * s["w_pre"]
    dh = s["dh"].float() + inv_h * (t - xh * (t * xh).mean(1, keepdim=True))
    du = dh * gate * wp
    db = inv_b * (du - xb * (du * xb).mean(1, keepdim=True)) if c["post"] else du
    got += [db.to(dt), (c["scale"] * dh).to(dt), (dy * xh).sum(0)]
    if c["post"]:
        got.append((dh * gate * xb).sum(0))
    if s["gate"] is not None:
        dg = dh * xb * wp
        got.append(dg.sum(0) if c["gate"] == "vector" else dg.to(dt))
    return got


def _plain_clip(s):
    # the arena holds nothing but the tensors (and zeros between them)
    g = s["raw"].float()
    norm = torch.sqrt((g * g).sum(dtype=torch.float64)).float()
    coef = torch.clamp(s["case"]["max_norm"] / (norm + 1e-6), max=1.0)
    return (g * coef).to(s["raw"].dtype), torch.stack((norm, coef))


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "attn":
        return _plain_attn(state)
    if kind == "rope":
        y = _plain_turn(state["x"], state, 1.0)
        return (y, _plain_turn(state["dy"], state, -1.0)) if state["case"]["direction"] == "step" else y
    return _plain_norm(state) if kind == "norm" else _plain_clip(state)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda t: t.to(torch.float64)  # noqa: E731
    step, back = case["direction"] == "step", case["direction"] == "backward"
    if case["kind"] == "attn":
        ql, kl = _lengths(case)
        per, d = case["heads"] // case["kv_heads"], case["head_dim"]
        out, dq = (torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        lse = torch.zeros((case["heads"], s["q"].shape[0]), dtype=torch.float64, device="cuda")
        q0 = 0
        for b, (nq, nk) in enumerate(zip(ql, kl)):
            k0 = b * case["capacity"] if case["capacity"] else sum(kl[:b])
            qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
            q0 += nq
            hidden = torch.zeros((nq, nk), dtype=torch.bool, device="cuda")
            if case["causal"]:
                hidden = torch.ones((nq, nk), dtype=torch.bool, device="cuda").triu(nk - nq + 1)
            for j in range(case["heads"]):
                q, k, v = f64(s["q"][qs, j]), f64(s["k"][ks, j // per]), f64(s["v"][ks, j // per])
                score = (q @ k.T / d ** 0.5).masked_fill(hidden, -math.inf)
                lse[j, qs] = torch.logsumexp(score, 1)
                p = torch.nan_to_num(torch.softmax(score, 1), nan=0.0)
                out[qs, j] = p @ v
                if step:
                    do = f64(s["dout"][qs, j])
                    dp = do @ v.T
                    ds = p * (dp - (do * out[qs, j]).sum(1, keepdim=True)) / d ** 0.5
                    dq[qs, j] = ds @ k
                    dk[ks, j // per] += ds.T @ q
                    dv[ks, j // per] += p.T @ do
        return (out, lse, dq, dk, dv) if step else (out, lse)
    if case["kind"] == "rope":
        turn = torch.polar(torch.full((case["rows"], len(s["frequencies"])), float(s["factor"]), dtype=torch.float64, device="cuda"),
                           f64(s["positions"])[:, None] * s["frequencies"])[:, None]

        def turned(x, by):
            x, dim = f64(x).clone(), case["rotary_dim"]
            at = (slice(0, dim, 2), slice(1, dim, 2)) if case["interleaved"] else (slice(0, dim // 2), slice(dim // 2, dim))
            z = torch.complex(x[..., at[0]], x[..., at[1]]) * by
            x[..., at[0]], x[..., at[1]] = z.real, z.imag
            return x
        return (turned(s["x"], turn), turned(s["dy"], turn.conj())) if step else turned(s["x"], turn)
    if case["kind"] == "norm":
        # the gradients by automatic differentiation of the definition
        leaf = lambda t: None if t is None else f64(t).requires_grad_()  # noqa: E731
        b, r, wp, gate, w = (leaf(s[n]) for n in ("b", "r", "w_post", "gate", "w_pre"))
        unit = lambda t: t / torch.sqrt(t.square().mean(1, keepdim=True) + s["eps"])  # noqa: E731
        branch = b if wp is None else unit(b) * wp
        h = case["scale"] * r + (branch if gate is None else branch * gate)
        # a backward pass is given h: the value at which the second norm is taken, whatever it was made from
        at = leaf(s["h"]) if back else h
        y = unit(at) * w
        if not (step or back):
            return [h.detach(), y.detach()]
        if back:
            dat, dw = torch.autograd.grad(y, (at, w), f64(s["dy"]))
            given, total = [h], [f64(s["dh"]) + dat]
        else:
            given, total = [h, y], [f64(s["dh"]), f64(s["dy"])]
        names = [b, r] + ([] if back else [w]) + [t for t in (wp, gate) if t is not None]
        g = list(torch.autograd.grad(given, names, total))
        g = g[:2] + [dw] + g[2:] if back else g
        return g if back else [h.detach(), y.detach()] + g
    g = f64(s["raw"])
    norm = torch.linalg.vector_norm(g)
    coef = min(1.0, case["max_norm"] / (float(norm) + 1e-6))
    return g * coef, torch.stack((norm, torch.full_like(norm, coef)))
