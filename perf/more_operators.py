"""Performance cases of a decoder's paged cache: attention of new tokens over it, the norms and rotation of queries
and keys with and without the writing of its pages, and the copying of pages.

A case is a dict of plain values.  "kind" is attn, qk, append or copy; "direction" of qk is forward or step
(forward, then backward).  New tokens and lengths of sequences are texts of whole numbers with commas between them;
a sequence without either is a place of the batch that no request has.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _attn(name, dtype, new, lengths, heads, kv_heads, head_dim, page, causal=True):
    """new: the queries of every sequence, the last of its `lengths` keys."""
    return {"name": name, "kind": "attn", "dtype": dtype, "new": ",".join(map(str, new)), "lengths": ",".join(map(str, lengths)),
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "causal": causal}


def _qk(name, dtype, rows, heads, kv_heads, head_dim, rotary_dim, interleaved, norm, far, direction="forward"):
    return {"name": name, "kind": "qk", "dtype": dtype, "direction": direction, "rows": rows, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rotary_dim": rotary_dim, "interleaved": interleaved, "norm": norm, "far": far}


def _append(name, dtype, new, lengths, heads, kv_heads, head_dim, rotary_dim, interleaved, norm, page):
    return {"name": name, "kind": "append", "dtype": dtype, "new": ",".join(map(str, new)), "lengths": ",".join(map(str, lengths)),
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "rotary_dim": rotary_dim, "interleaved": interleaved,
            "norm": norm, "page": page}


def _copy(name, dtype, count, pages, planes, page, kv_heads, head_dim):
    """planes: keys and values of each layer."""
    return {"name": name, "kind": "copy", "dtype": dtype, "count": count, "pages": pages, "planes": planes, "page": page,
            "kv_heads": kv_heads, "head_dim": head_dim}


def listed():
    held = [16384, 12001, 9000, 8192, 6001, 5120, 4097, 4096, 3500, 2777, 2048, 1999, 1024, 700, 513, 300, 128, 77, 64, 17, 1, 0, 0, 0]
    some = [6000, 5501, 4096, 3333, 2500, 1500, 1025, 1024, 800, 400, 399, 256, 90, 33, 8, 1, 0]
    return [
        # answering: one new token for each request, over caches that are filled unevenly; the batch is not full
        _attn("attn_token", "bf16", [min(n, 1) for n in held], held, 32, 8, 128, 16),
        # the smallest call: one token of one request
        _attn("attn_one", "bf16", [1], [777], 32, 8, 128, 16),
        # prompts that come in chunks: the next chunk of each over what its earlier ones left, the last one just begun
        _attn("attn_chunk", "bf16", [2048, 1024, 777, 513], [8192, 5021, 9999, 513], 32, 8, 128, 16),
        # one chunk of a prompt among requests that are answered token by token
        _attn("attn_mixed", "bf16", [256] + [min(n, 1) for n in some], [5000] + some, 28, 4, 128, 32),
        # chunks in fp32
        _attn("attn_chunk_f32", "f32", [512, 301, 64, 1], [2048, 1301, 4000, 777], 16, 4, 64, 64),
        # queries and keys of one new token a request
        _qk("qk_token", "bf16", 16, 32, 8, 128, 128, False, True, 131072),
        # ... of a training step
        _qk("qk_train", "bf16", 16381, 32, 8, 128, 128, False, True, 16384, "step"),
        # ... in fp32 with odd sizes, half of each head turned, pairs side by side
        _qk("qk_step_f32", "f32", 4095, 15, 5, 80, 40, True, True, 4096, "step"),
        # the new tokens of a full batch of requests go to the cache
        _append("append_token", "bf16", [1] * 48, [1 + 97 * i for i in range(48)], 32, 8, 128, 128, False, True, 16),
        # ... and those of packed prompts
        _append("append_prompt", "bf16", [4096, 3333, 2900, 1531, 640, 97], [4096, 8001, 2900, 9000, 640, 777], 32, 8, 128, 128, False, True, 16),
        # requests that share a prefix take a copy of its last page each, in every layer
        _copy("copy_fork", "bf16", 5, 256, 24, 16, 8, 128),
        # the pages in use move together
        _copy("copy_compact", "bf16", 600, 1500, 32, 16, 8, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    most = {}
    for c in listed():
        w = work(c)
        f, b = most.get(c["kind"], (0, 0))
        most[c["kind"]] = (max(f, w["flops"]), max(b, w["bytes"]))
    kind = rng.choice(["attn", "attn", "attn", "qk", "append", "copy"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        kv = rng.choice([1, 2, 3, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 3, 4, 7, 8])
        dim = rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
        rotary, page = rng.choice([dim, dim, dim // 2]), rng.choice([8, 16, 16, 32, 64, 128])
        far = rng.choice(["token", "chunk", "mixed"])
        n = _log_int(rng, 1, 48 if far == "token" else 12)
        lengths = [_log_int(rng, 1, 16384 if far == "token" else 8192) for _ in range(n)]
        new = [1 if far == "token" or (far == "mixed" and i % 3) else _log_int(rng, 1, min(k, 2048)) for i, k in enumerate(lengths)]
        if rng.random() < 0.3:  # a place without a request
            new, lengths = new + [0], lengths + [0]
        if kind == "attn":
            if rng.random() < 0.1:  # more queries than keys: the first see nothing
                new[0] = lengths[0] + rng.randint(1, 5)
            c = _attn("", dtype, new, lengths, heads, kv, dim, page, rng.random() < 0.85)
        elif kind == "qk":
            c = _qk("", dtype, _log_int(rng, 1, 16381), heads, kv, dim, rotary, rng.random() < 0.5, rng.random() < 0.8, _log_int(rng, 64, 131072),
                    rng.choice(["forward", "step"]))
        elif kind == "append":
            c = _append("", dtype, new, lengths, heads, kv, dim, rotary, rng.random() < 0.5, rng.random() < 0.8, page)
        else:
            count = _log_int(rng, 1, 600)
            c = _copy("", dtype, count, 2 * count + rng.randint(1, 300), 2 * rng.randint(1, 16), page, kv, dim)
        w = work(c)
        padded = 1
        if kind == "attn":
            padded = len(new) * max(new) * max(lengths) * heads / (4 * 2048 * 9999 * 32)
        elif kind == "copy":
            padded = c["pages"] * c["planes"] * page * kv * dim * 2 / 2 ** 32
        # fp32 products of matrices are a sixteenth as fast
        if w["flops"] * (16 if dtype == "f32" and kind == "attn" else 1) <= most[kind][0] and w["bytes"] <= most[kind][1] and padded <= 1:
            del c["name"]
            return c


# ---------------------------------------------------------------- sizes

def _numbers(case):
    return [int(v) for v in case["new"].split(",")], [int(v) for v in case["lengths"].split(",")]


def _pairs(nq, nk, causal):
    """How many (query, key) pairs see each other; query i of nq sees keys up to i + nk - nq."""
    if not causal:
        return nq * nk
    first = max(0, nq - nk)  # queries before this one see nothing
    n = nq - first
    return n * (nk - nq + first + 1) + n * (n - 1) // 2


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "copy":
        return {"bytes": 2 * case["count"] * case["planes"] * case["page"] * case["kv_heads"] * case["head_dim"] * size, "flops": 0}
    h, g, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "attn":
        new, lengths = _numbers(case)
        nq = sum(new)
        pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(new, lengths)) * h
        pages = sum(-(-n // case["page"]) for n, q in zip(lengths, new) if q)
        # queries read, out and the rows' log sums written, each key and value that is seen read once, and their pages' numbers
        keys = sum(n for n, q in zip(lengths, new) if q)
        return {"bytes": (2 * nq * h + 2 * keys * g) * d * size + 4 * nq * h + 4 * pages, "flops": 4 * d * pairs}
    if case["kind"] == "qk":
        n = case["rows"] * (h + g) * d
        step = case["direction"] == "step"
        return {"bytes": (5 if step else 2) * n * size + (2 if step else 1) * 4 * case["rows"], "flops": (24 if step else 8) * n}
    n = sum(_numbers(case)[0])
    return {"bytes": 2 * n * (h + 2 * g) * d * size + 4 * n, "flops": 8 * n * (h + g) * d}


# ---------------------------------------------------------------- inputs

def _rand(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _turning(case):
    """Turning angle per position of each pair, in double precision."""
    dim = case["rotary_dim"]
    return torch.tensor(10000.0 ** (-np.arange(0, dim, 2, dtype=np.float64) / dim), device="cuda")


def _cache(s, gen, case, dt):
    """A pool of pages, some of which no sequence has, and each sequence's pages in the order of its tokens."""
    new, lengths = _numbers(case)
    page = case["page"]
    need = [-(-n // page) for n in lengths]
    s["pages"], s["columns"] = sum(need) + 7, max(max(need), 1)
    shape = (s["pages"], page, case["kv_heads"], case["head_dim"])
    s["k_pages"], s["v_pages"] = _rand(gen, shape, dt), _rand(gen, shape, dt)
    order = torch.randperm(s["pages"], generator=gen, device="cuda").to(torch.int32)
    places = np.concatenate([[0], np.cumsum(need)])
    at = np.minimum(places[:-1, None] + np.arange(s["columns"])[None, :], s["pages"] - 1)
    used = np.arange(s["columns"])[None, :] < np.asarray(need)[:, None]
    s["table"] = torch.where(torch.tensor(used, device="cuda"), order[torch.tensor(at, device="cuda")], torch.full((), -1, dtype=torch.int32, device="cuda"))
    s["q_offsets"], s["lengths"] = _ints(np.cumsum([0] + new)), _ints(lengths)
    s["rows"], s["max_q"], s["max_k"] = sum(new), max(new), max(lengths)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "copy":
        s["pool"] = _rand(gen, (case["planes"], case["pages"], case["page"] * case["kv_heads"] * case["head_dim"]), dt)
        s["pairs"] = torch.randperm(case["pages"], generator=gen, device="cuda")[:2 * case["count"]].reshape(-1, 2).to(torch.int32)
    else:
        h, g, d = case["heads"], case["kv_heads"], case["head_dim"]
        if case["kind"] == "qk":
            s["rows"] = case["rows"]
        else:
            _cache(s, gen, case, dt)
        n = s["rows"]
        if case["kind"] == "attn":
            s["q"] = _rand(gen, (n, h, d), dt)
        else:
            # queries, keys and values lie side by side in the rows of one product
            s["x"] = _rand(gen, (n, (h + 2 * g) * d), dt, 1.5)
            s["q"], s["k"], s["v"] = s["x"].split([h * d, g * d, g * d], 1)
            s["w_q"], s["w_k"] = ((1 + _rand(gen, (d,), torch.float32, 0.2)) if case["norm"] else None for _ in range(2))
            s["frequencies"], s["eps"], s["factor"] = _turning(case), 1e-6, 1.0
        if case["kind"] == "qk":
            s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
            s["dq_out"], s["dk_out"] = _rand(gen, (n, h, d), dt), _rand(gen, (n, g, d), dt)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """Plans, outputs and workspaces, which a user's program makes once and keeps."""
    import paper_1707_06990_amd as dnb
    c = s["case"]
    dt = dnb.DNB_F32 if c["dtype"] == "f32" else dnb.DNB_BF16
    s["dnb"] = dnb
    if c["kind"] == "copy":
        return
    h, g, d, n = c["heads"], c["kv_heads"], c["head_dim"], s["rows"]
    room = lambda k: torch.empty(max(16, k), dtype=torch.uint8, device="cuda")  # noqa: E731
    if c["kind"] != "qk":
        s["cache"] = dnb.dnb_paged_layout(s["pages"], c["page"], g, d, s["lengths"].numel(), s["columns"], dtype=dt)
    if c["kind"] == "attn":
        s["plan"] = dnb.dnb_paged_attn_create(s["cache"], h, n, causal=c["causal"])
        s["workspace"] = room(dnb.dnb_paged_attn_workspace_bytes(s["plan"]))
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((h, n), device="cuda")
        return
    s["turns"] = s["frequencies"] / (2 * math.pi)
    stride = s["x"].shape[1]
    order = dnb.DNB_ROPE_INTERLEAVED if c["interleaved"] else dnb.DNB_ROPE_HALF
    s["qk"] = dnb.dnb_qk_layout(n, h, g, d, c["rotary_dim"], order, dtype=dt, eps=s["eps"], factor=s["factor"], q_stride=stride, k_stride=stride,
                                v_stride=stride)
    s["q_out"], s["k_out"] = (torch.empty((n, m, d), dtype=s["x"].dtype, device="cuda") for m in (h, g))
    if c["kind"] == "qk" and c["direction"] == "step":
        s["dx"] = torch.empty_like(s["x"])
        s["dq"], s["dk"], _ = s["dx"].split([h * d, g * d, g * d], 1)
        s["dw_q"], s["dw_k"] = (torch.empty_like(s["w_q"]) if c["norm"] else None for _ in range(2))
        s["scratch"] = room(dnb.dnb_op_qk_rope_scratch_bytes(s["qk"]))


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    dnb, c = s["dnb"], s["case"]
    if c["kind"] == "attn":
        dnb.dnb_paged_attn_forward(s["plan"], s["q"], s["k_pages"], s["v_pages"], s["q_offsets"], s["lengths"], s["table"], s["out"], s["lse"],
                                   s["workspace"])
        return s["out"], s["lse"]
    if c["kind"] == "append":
        dnb.dnb_op_paged_append(s["qk"], s["cache"], s["q"], s["k"], s["v"], s["w_q"], s["w_k"], None, s["turns"], s["q_offsets"], s["lengths"],
                                s["table"], s["q_out"], s["k_pages"], s["v_pages"])
        return s["q_out"], s["k_pages"], s["v_pages"]
    if c["kind"] == "copy":
        pool = s["pool"]
        nbytes = pool.shape[2] * pool.element_size()
        dnb.dnb_op_paged_copy(pool, c["pages"], nbytes, c["planes"], c["pages"] * nbytes, s["pairs"], c["count"])
        return pool
    dnb.dnb_op_qk_rope_forward(s["qk"], s["q"], s["k"], s["w_q"], s["w_k"], s["positions"], s["turns"], s["q_out"], s["k_out"])
    if c["direction"] != "step":
        return s["q_out"], s["k_out"]
    dnb.dnb_op_qk_rope_backward(s["qk"], s["q"], s["k"], s["w_q"], s["w_k"], s["positions"], s["turns"], s["dq_out"], s["dk_out"], s["dq"], s["dk"],
                                s["dw_q"], s["dw_k"], s["scratch"])
    return [t for t in (s["q_out"], s["k_out"], s["dq"], s["dk"], s["dw_q"], s["dw_k"]) if t is not None]


# ---------------------------------------------------------------- the plain forms

def _places(s):
    """Of every new token: its sequence and its place there."""
    o = s["q_offsets"].long()
    new = o[1:] - o[:-1]
    seq = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=s["rows"])
    return seq, torch.arange(s["rows"], device="cuda") - o[seq], new


def _plain_attn(s):
    c = s["case"]
    h, g, d, page = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    per, dt = h // g, s["q"].dtype
    seq, at, new = _places(s)
    n, mq, mk = new.numel(), s["max_q"], s["max_k"]
    lengths = s["lengths"].long()
    # the cache's rows of every sequence side by side, those past its length on the pool's first
    key = torch.arange(mk, device="cuda")
    real_k = key[None, :] < lengths[:, None]
    rows_k = torch.where(real_k, s["table"].long()[:, key // page] * page + key % page, torch.zeros_like(real_k, dtype=torch.long))
    keys, values = (t.reshape(-1, g, d)[rows_k].float().transpose(1, 2) for t in (s["k_pages"], s["v_pages"]))
    query = torch.arange(mq, device="cuda")
    real_q = query[None, :] < new[:, None]
    rows_q = torch.where(real_q, s["q_offsets"].long()[:-1, None] + query[None, :], torch.zeros_like(real_q, dtype=torch.long))
    q = s["q"][rows_q].float().transpose(1, 2).reshape(n, g, per * mq, d)
    seen = real_q[:, :, None] & real_k[:, None, :]
    if c["causal"]:
        seen &= key[None, None, :] <= (query[None, :] + (lengths - new)[:, None])[:, :, None]
    seen = seen[:, None, None].expand(n, g, per, mq, mk).reshape(n, g, per * mq, mk) if per > 1 else seen[:, None]
    p = (q @ keys.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(d)).masked_fill_(~seen, -math.inf)
    top = p.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(p.sub_(top))
    total = p.sum(3, keepdim=True)
    lse = (torch.log(total) + top).reshape(n, h, mq).transpose(1, 2)[seq, at].transpose(0, 1).contiguous()
    out = (p @ values.contiguous()) / torch.where(total == 0, torch.ones_like(total), total)
    return out.reshape(n, h, mq, d).transpose(1, 2)[seq, at].to(dt), lse


def _angles(s, positions):
    """Cosine and sine of every (row, pair); far positions need more than 32 bits."""
    angle = positions.double()[:, None] * s["frequencies"][None, :]
    return (torch.cos(angle) * s["factor"]).float()[:, None], (torch.sin(angle) * s["factor"]).float()[:, None]


def _turn(c, x, cos, sin):
    dim, half = c["rotary_dim"], c["rotary_dim"] // 2
    turned = x[..., :dim]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if c["interleaved"] else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).reshape(turned.shape) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., dim:]), -1)


def _unit(s, x):
    """x in 32 bits over its root mean square, and one over that."""
    x = x.float().reshape(x.shape[0], -1, s["case"]["head_dim"])
    inv = torch.rsqrt((x * x).mean(2, keepdim=True) + s["eps"])
    return x * inv, inv


def _plain_heads(s, x, w, cos, sin):
    y = x.float().reshape(x.shape[0], -1, s["case"]["head_dim"]) if w is None else _unit(s, x)[0] * w
    return _turn(s["case"], y, cos, sin).to(x.dtype)


def _plain_gradients(s, x, w, dy, cos, sin):
    dn = _turn(s["case"], dy.float(), cos, -sin)
    if w is None:
        return dn.to(x.dtype).reshape(x.shape), None
    unit, inv = _unit(s, x)
    t = dn * w
    dx = inv * (t - unit * (t * unit).mean(2, keepdim=True))
    return dx.to(x.dtype).reshape(x.shape), (dn * unit).sum((0, 1))


def _plain_qk(s):
    cos, sin = _angles(s, s["positions"])
    got = [_plain_heads(s, s["q"], s["w_q"], cos, sin), _plain_heads(s, s["k"], s["w_k"], cos, sin)]
    if s["case"]["direction"] != "step":
        return tuple(got)
    dq, dw_q = _plain_gradients(s, s["q"], s["w_q"], s["dq_out"], cos, sin)
    dk, dw_k = _plain_gradients(s, s["k"], s["w_k"], s["dk_out"], cos, sin)
    return [t for t in (*got, dq, dk, dw_q, dw_k) if t is not None]


def _plain_append(s):
    c = s["case"]
    seq, at, new = _places(s)
    place = at + (s["lengths"].long() - new)[seq]
    cos, sin = _angles(s, place)
    row = s["table"].long()[seq, place // c["page"]] * c["page"] + place % c["page"]
    s["k_pages"].view(-1, c["kv_heads"], c["head_dim"])[row] = _plain_heads(s, s["k"], s["w_k"], cos, sin)
    s["v_pages"].view(-1, c["kv_heads"], c["head_dim"])[row] = s["v"].reshape(-1, c["kv_heads"], c["head_dim"])
    return _plain_heads(s, s["q"], s["w_q"], cos, sin), s["k_pages"], s["v_pages"]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "copy":
        pairs = state["pairs"].long()
        state["pool"][:, pairs[:, 1]] = state["pool"][:, pairs[:, 0]]
        return state["pool"]
    return _plain_attn(state) if kind == "attn" else _plain_qk(state) if kind == "qk" else _plain_append(state)


# ---------------------------------------------------------------- the definitions in 64 bits

def _spun(case, s, x, positions, by):
    """Heads of x turned by the positions, in either direction."""
    turn = torch.polar(torch.full((x.shape[0], s["frequencies"].numel()), float(s["factor"]), dtype=torch.float64, device="cuda"),
                       by * positions.double()[:, None] * s["frequencies"])[:, None]
    dim = case["rotary_dim"]
    first, second = (slice(0, dim, 2), slice(1, dim, 2)) if case["interleaved"] else (slice(0, dim // 2), slice(dim // 2, dim))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda t: None if t is None else t.detach().to(torch.float64)  # noqa: E731
    if case["kind"] == "copy":
        pool = f64(s["pool"])
        for a, b in s["pairs"].tolist():
            pool[:, b] = f64(s["pool"][:, a])
        return pool
    h, g, d = case["heads"], case["kv_heads"], case["head_dim"]

    def heads(x, w, m, positions):
        x = x.reshape(-1, m, d)
        if w is not None:
            x = x / torch.sqrt(x.square().sum(2, keepdim=True) / d + s["eps"]) * w
        return _spun(case, s, x, positions, 1.0)
    if case["kind"] == "qk":
        got, grads, weights = [], [], []
        for x, w, m, dy in ((s["q"], s["w_q"], h, s["dq_out"]), (s["k"], s["w_k"], g, s["dk_out"])):
            x, w = f64(x).requires_grad_(), None if w is None else f64(w).requires_grad_()
            if case["direction"] == "step":
                # the gradients by automatic differentiation of the norm, of what the rotation hands back
                back = _spun(case, s, f64(dy), s["positions"], -1.0)
                y = x.reshape(-1, m, d)
                y = y if w is None else y / torch.sqrt(y.square().sum(2, keepdim=True) / d + s["eps"]) * w
                found = torch.autograd.grad(y, [x] if w is None else [x, w], back)
                grads.append(found[0])
                weights += found[1:]
            with torch.no_grad():
                got.append(heads(x.detach(), None if w is None else w.detach(), m, s["positions"]))
        return got + grads + weights if case["direction"] == "step" else tuple(got)
    new, lengths = _numbers(case)
    table, page = s["table"].cpu().numpy(), case["page"]
    # rows of the pool in the order of each sequence's tokens
    row = lambda b, places: torch.tensor(table[b, places // page].astype(np.int64) * page + places % page, device="cuda")  # noqa: E731
    if case["kind"] == "append":
        first = [n - q for n, q in zip(lengths, new)]
        positions = torch.tensor(np.concatenate([np.arange(a, n) for a, n in zip(first, lengths)]), device="cuda")
        rows = torch.cat([row(b, np.arange(a, n)) for b, (a, n) in enumerate(zip(first, lengths))])
        k_pages, v_pages = f64(s["k_pages"]), f64(s["v_pages"])
        k_pages.view(-1, g, d)[rows] = heads(f64(s["k"]), f64(s["w_k"]), g, positions)
        v_pages.view(-1, g, d)[rows] = f64(s["v"]).reshape(-1, g, d)
        return heads(f64(s["q"]), f64(s["w_q"]), h, positions), k_pages, v_pages
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((h, s["rows"]), dtype=torch.float64, device="cuda")
    q0 = 0
    for b, (nq, nk) in enumerate(zip(new, lengths)):
        qs = slice(q0, q0 + nq)
        q0 += nq
        if nq == 0:
            continue
        rows = row(b, np.arange(nk))
        hidden = torch.zeros((nq, nk), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = torch.ones((nq, nk), dtype=torch.bool, device="cuda").triu(nk - nq + 1)
        for j in range(h):
            k, v = (f64(t.view(-1, g, d)[rows, j // (h // g)]) for t in (s["k_pages"], s["v_pages"]))
            score = (f64(s["q"][qs, j]) @ k.T / d ** 0.5).masked_fill(hidden, -math.inf)
            lse[j, qs] = torch.logsumexp(score, 1)
            out[qs, j] = torch.nan_to_num(torch.softmax(score, 1), nan=0.0) @ v
    return out, lse
