"""Which kernels an attention plan runs, by the rules beside them, so that a test says which form it is for."""


def split_rows(rq, rk, n, kv, per, bf16):
    """The work of few rows is split over the keys (forward and dq)."""
    tiles = (rq * per // 128 + n) * kv
    return (rq * per <= 32 * n or tiles <= (40 if bf16 else 96)) and 2 * rk >= (n + 1) * (400 if bf16 else 256)


def form(dtype, q_lengths, rows_k, heads, kv_heads):
    """"split", or tiles of 128 rows by "four" or "eight" waves."""
    rq, n, per = sum(q_lengths), len(q_lengths), heads // kv_heads
    if split_rows(rq, rows_k, n, kv_heads, per, dtype == "bf16"):
        return "split"
    tiles = (rq * per + 127) // 128 + n
    return "eight" if tiles * kv_heads <= 256 and rows_k >= 256 * n else "four"


def check(dnb, p, want):
    """That Problem p runs that form; the split one shows in the plan's workspace too."""
    dtype = "bf16" if "bfloat16" in str(p.dt) else "f32"
    q = [b - a for a, b in zip(p.qo, p.qo[1:])]
    heads, kv, dim = p.q.shape[1], p.k.shape[1], p.q.shape[2]
    assert form(dtype, q, p.k.shape[0], heads, kv) == want
    # partial results of 2048 (fp32 1024) waves, 32 rows of head_dim each
    parts = (2048 if dtype == "bf16" else 1024) * 32 * 4 * (-(-dim // 32) * 32)
    if want == "split":
        assert dnb.dnb_attn_workspace_bytes(p.plan) >= 4 * sum(q) * heads + parts
