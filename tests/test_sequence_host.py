"""CPU-side checks of the sequence operators: what their plans and entry points refuse, before any launch."""
import ctypes

import pytest

ATTN = dict(heads=8, kv_heads=2, head_dim=64, sequences=3, rows_q=100, rows_k=200)


def status(call):
    """0, or the status with which it was refused."""
    import paper_1707_06990_amd as dnb
    try:
        call()
        return 0
    except dnb.DnbError as e:
        return e.status


@pytest.mark.parametrize("kw,code", [
    (dict(heads=0), -1), (dict(kv_heads=0), -1), (dict(heads=7), -1), (dict(head_dim=0), -1), (dict(sequences=0), -1),
    (dict(rows_q=-1), -1), (dict(rows_k=-1), -1), (dict(dtype=5), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(head_dim=36), -5), (dict(head_dim=136), -5),
    (dict(q_stride=504), -6), (dict(k_stride=120), -6), (dict(v_stride=132), -6), (dict(k_stride=-128), -6), (dict(k_stride=(1 << 22) + 8), -6),
    (dict(rows_q=2 ** 31), -6), (dict(rows_k=2 ** 31), -6), (dict(rows_q=2 ** 30, heads=8, kv_heads=1), -6), (dict(heads=1 << 17), -6),
    (dict(rows_q=2 ** 28, heads=64, kv_heads=64), -6), (dict(sequences=1 << 21), -6)])
def test_attention_plans_that_are_refused(dnb, kw, code):
    assert status(lambda: dnb.dnb_attn_create(**{**ATTN, **kw})) == code


@pytest.mark.parametrize("kw", [{}, dict(rows_q=0), dict(rows_k=0), dict(heads=2), dict(head_dim=8), dict(head_dim=128), dict(dtype=0),
                                dict(q_stride=768, k_stride=768, v_stride=768), dict(dtype=0, k_stride=132), dict(rows_k=2 ** 31 - 1)])
def test_attention_plans_that_are_taken(dnb, kw):
    p = dnb.dnb_attn_create(**{**ATTN, **kw})
    rows, heads = {**ATTN, **kw}["rows_q"], {**ATTN, **kw}["heads"]
    assert dnb.dnb_attn_workspace_bytes(p) >= 4 * rows * heads
    dnb.dnb_attn_destroy(p)


def test_attention_arguments(dnb):
    lib = ctypes.CDLL(dnb.binding.LIB_PATH)
    fwd, bwd = lib.dnb_attn_forward, lib.dnb_attn_backward
    fwd.argtypes, bwd.argtypes = [ctypes.c_void_p] * 11, [ctypes.c_void_p] * 15
    p = dnb.dnb_attn_create(**ATTN)
    ok = [4096 * (i + 1) for i in range(12)]
    for missing in (0, 1, 2, 3, 4, 6, 7, 8):   # (k_lengths, 5, may be null)
        args = [None if i == missing else ok[i] for i in range(9)]
        assert fwd(p, *args, None) == -2, missing
    for odd in (0, 1, 2, 6, 8):
        args = [ok[i] + 8 if i == odd else ok[i] for i in range(9)]
        assert fwd(p, *args, None) == -3, odd
    assert fwd(None, *ok[:9], None) == -2
    for missing in (0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11):   # (k_lengths: 8)
        args = [None if i == missing else ok[i] for i in range(12)] + [65536]
        assert bwd(p, *args, None) == -2, missing
    assert bwd(p, *ok, None, None) == -2
    for odd in (0, 1, 2, 3, 5, 9, 10, 11):
        args = [ok[i] + 4 if i == odd else ok[i] for i in range(12)] + [65536]
        assert bwd(p, *args, None) == -3, odd
    dnb.dnb_attn_destroy(p)
    assert lib.dnb_attn_create(None, None) == -2
    # nothing to do: no launch, no pointers looked at but the offsets
    p = dnb.dnb_attn_create(**{**ATTN, "rows_q": 0})
    assert fwd(p, None, None, None, 4096, 4096, None, None, None, None, None) == 0
    dnb.dnb_attn_destroy(p)
