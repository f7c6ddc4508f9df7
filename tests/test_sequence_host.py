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


@pytest.mark.parametrize("kw,code", [
    (dict(order=2), -1), (dict(dtype=3), -1), (dict(rows=-1), -1), (dict(heads=0), -1), (dict(head_dim=63), -1), (dict(rotary_dim=7), -1),
    (dict(rotary_dim=66), -1), (dict(rotary_dim=0), -1), (dict(heads=4097), -6), (dict(head_dim=1026), -6), (dict(x_stride=100), -6),
    (dict(y_stride=513), -6), (dict(x=None), -2), (dict(positions=None), -2), (dict(turns=None), -2), (dict(y=None), -2),
    (dict(x=4104), -3), (dict(y=4100), -3), (dict(positions=4098), -3), (dict(turns=4100), -3), (dict(rows=0, x=None), 0)])
def test_rotary_arguments(dnb, kw, code):
    base = dict(x=4096, positions=8192, turns=12288, y=16384, rows=4, heads=8, head_dim=64, rotary_dim=64, order=dnb.DNB_ROPE_HALF, factor=1.0,
                dtype=dnb.DNB_BF16, stream=0)
    args = {**base, **kw}
    assert status(lambda: dnb.dnb_op_rope_forward(**args)) == code
    names = dict(x="dy", y="dx", x_stride="dy_stride", y_stride="dx_stride")
    assert status(lambda: dnb.dnb_op_rope_backward(**{names.get(k, k): v for k, v in args.items()})) == code


@pytest.mark.parametrize("kw,code", [
    (dict(gate_kind=3), -1), (dict(dtype=2), -1), (dict(rows=-1), -1), (dict(width=0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(scale=float("nan")), -1), (dict(width=60), -5), (dict(width=16392), -6), (dict(b=None), -2), (dict(w_pre=None), -2),
    (dict(gate=None), -2), (dict(b=4104), -3), (dict(w_post=4100), -3), (dict(gate=4098), -3)])
def test_norm_arguments(dnb, kw, code):
    p = iter(range(4096, 4096 * 30, 4096))
    base = dict(b=next(p), w_post=next(p), gate=next(p), w_pre=next(p), rows=4, width=64, scale=1.0, eps=1e-6, gate_kind=dnb.DNB_GATE_VECTOR,
                dtype=dnb.DNB_F32, stream=0)
    fwd = dict(r=next(p), h_new=next(p), y=next(p))
    back = dict(h_new=next(p), dh=next(p), dy=next(p), db=next(p), dr=next(p), dw_post=next(p), dgate=next(p), dw_pre=next(p), scratch=next(p))
    assert status(lambda: dnb.dnb_op_norm_residual_forward(**{**base, **fwd, **kw})) == code
    assert status(lambda: dnb.dnb_op_norm_residual_backward(**{**base, **back, **kw})) == code
    for n in ("r", "h_new", "y"):
        assert status(lambda: dnb.dnb_op_norm_residual_forward(**{**base, **fwd, n: None})) == -2
    for n in back:
        assert status(lambda: dnb.dnb_op_norm_residual_backward(**{**base, **back, n: None})) == -2
        assert status(lambda: dnb.dnb_op_norm_residual_backward(**{**base, **back, n: back[n] + 4})) == -3
    assert dnb.dnb_op_norm_residual_scratch_bytes(4, 60, 0) == 0
    assert dnb.dnb_op_norm_residual_scratch_bytes(10, 64, 1) >= 2 * 64 * 4


def test_clipping_plans(dnb):
    make = lambda src, dst, types, counts: dnb.dnb_clip_create(src, dst, types, counts)
    assert status(lambda: make([4096], [None], [0], [5])) == -2
    assert status(lambda: make([None], [4096], [0], [5])) == -2
    assert status(lambda: make([4096], [4096], [2], [5])) == -1
    assert status(lambda: make([4096], [4096], [0], [-1])) == -1
    assert status(lambda: make([4098], [4096], [0], [5])) == -3
    assert status(lambda: make([4096], [4097], [1], [5])) == -3
    assert status(lambda: make([4096], [4096], [0], [2 ** 50])) == -6
    with pytest.raises(ValueError):
        make([4096], [4096, 8192], [0], [5])
    plan = make([None, 4096, 1 << 20], [None, 4096, 1 << 21], [0, 1, 0], [0, 16384, 40000])
    assert dnb.dnb_clip_table(plan).size == dnb.dnb_clip_table_bytes(plan) == 24 * 4   # 1 + 3 parts of 16384 values
    assert dnb.dnb_clip_workspace_bytes(plan) == 8 * 4
    run = lambda **kw: dnb.dnb_clip_run(**{**dict(plan=plan, table=4096, max_norm=1.0, norm=8192, workspace=12288, stream=0), **kw})
    for kw, code in ((dict(max_norm=-1.0), -1), (dict(max_norm=float("nan")), -1), (dict(table=None), -2), (dict(norm=None), -2),
                     (dict(workspace=None), -2), (dict(plan=None), -2), (dict(table=4104), -3), (dict(workspace=4100), -3), (dict(norm=4098), -3)):
        assert status(lambda: run(**kw)) == code, kw
    dnb.dnb_clip_destroy(plan)
    empty = make([], [], [], [])
    assert dnb.dnb_clip_table(empty).size == 0
    dnb.dnb_clip_destroy(empty)
