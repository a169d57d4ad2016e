"""Argument checks of dp_attention, dp_group_norm and dp_group_norm_daq: found on the host, before anything is enqueued. No
GPU needed: every refusal comes before the library looks at the device (and no call here gets that far)."""
import ctypes as C

import pytest

from paper_2511_11446_b200 import binding as B

A = 1 << 20  # an aligned address that nobody dereferences


def _attn(**kw):
    f = dict(heads=4, kv_heads=2, head_dim=64, n_seq=2, max_q=10, max_k=20, scale=0.125)
    f.update(kw)
    a = B.dp_attn()
    for k, v in f.items():
        setattr(a, k, v)
    return a


def _call(a, q=A, ldq=256, Mq=20, k=2 * A, ldk=128, v=3 * A, ldv=128, Mk=40, y=4 * A, ldy=256, flags=0):
    return B.lib().dp_attention(C.byref(a) if a is not None else None, q, ldq, Mq, k, ldk, v, ldv, Mk, y, ldy, None, flags, None)


@pytest.mark.parametrize("want,fields,args", [
    (B.DP_ERR_SHAPE, dict(heads=0), {}),
    (B.DP_ERR_SHAPE, dict(heads=3), {}),                       # not a multiple of kv_heads
    (B.DP_ERR_SHAPE, dict(kv_heads=0), {}),
    (B.DP_ERR_SHAPE, dict(head_dim=4), {}),
    (B.DP_ERR_SHAPE, dict(head_dim=136), {}),
    (B.DP_ERR_SHAPE, dict(head_dim=60), {}),
    (B.DP_ERR_SHAPE, dict(n_seq=-1), {}),
    (B.DP_ERR_SHAPE, dict(max_q=-1), {}),
    (B.DP_ERR_SHAPE, dict(max_k=1 << 31), {}),
    (B.DP_ERR_SHAPE, dict(max_q=11), {}),                      # two sequences of 11 in 20 rows
    (B.DP_ERR_SHAPE, dict(max_k=21), {}),
    (B.DP_ERR_SHAPE, {}, dict(Mq=-1)),
    (B.DP_ERR_SHAPE, {}, dict(Mk=1 << 31)),
    (B.DP_ERR_INVALID_ARG, dict(q_start=A), {}),               # without k_start
    (B.DP_ERR_INVALID_ARG, dict(mask=2), {}),
    (B.DP_ERR_INVALID_ARG, dict(prefix=A), {}),                # without the causal mask
    (B.DP_ERR_INVALID_ARG, dict(scale=float("nan")), {}),
    (B.DP_ERR_INVALID_ARG, dict(scale=float("inf")), {}),
    (B.DP_ERR_INVALID_ARG, dict(scale=-1.0), {}),
    (B.DP_ERR_INVALID_ARG, dict(cap=-1.0), {}),
    (B.DP_ERR_INVALID_ARG, dict(cap=float("inf")), {}),
    (B.DP_ERR_INVALID_ARG, dict(cap=1e5), {}),
    (B.DP_ERR_SHAPE, {}, dict(ldq=56)),
    (B.DP_ERR_SHAPE, dict(k_head_stride=56), {}),
    (B.DP_ERR_SHAPE, dict(k_head_stride=-64), {}),
    (B.DP_ERR_SHAPE, {}, dict(ldk=1 << 39)),
    (B.DP_ERR_SHAPE, {}, dict(ldy=128)),                       # rows and heads of y overlap
    (B.DP_ERR_INVALID_ARG, {}, dict(q=None)),
    (B.DP_ERR_INVALID_ARG, {}, dict(k=None)),
    (B.DP_ERR_INVALID_ARG, {}, dict(v=None)),
    (B.DP_ERR_INVALID_ARG, {}, dict(y=None)),
    (B.DP_ERR_ALIGN, {}, dict(q=A + 2)),
    (B.DP_ERR_ALIGN, {}, dict(y=4 * A + 8)),
    (B.DP_ERR_ALIGN, {}, dict(ldv=130)),
    (B.DP_ERR_ALIGN, dict(v_head_stride=68), {}),
    (B.DP_ERR_ALIGN, dict(slopes=A + 2), {}),
    (B.DP_ERR_INVALID_ARG, {}, dict(y=A)),                     # y is q
    (B.DP_ERR_INVALID_ARG, {}, dict(y=2 * A + 128)),           # y reaches into k
    (B.DP_ERR_INVALID_ARG, {}, dict(y=A + 256, ldq=1024, ldy=1024)),   # columns of one buffer that meet
    (B.DP_ERR_INVALID_ARG, {}, dict(y=A + 504 * 2, ldq=512, ldy=512)),     # the last 8 reach into the next row's q
    (B.DP_ERR_INVALID_ARG, {}, dict(flags=0x10000)),
    (B.DP_ERR_INVALID_ARG, {}, dict(flags=B.DP_FLAG_FORCE_SIMT | B.DP_FLAG_FORCE_MMA)),
])
def test_attention_refusals(want, fields, args):
    assert _call(_attn(**fields), **args) == want
    assert B.lib().dp_last_error()


@pytest.mark.parametrize("fields,args", [
    ({}, dict(Mq=1 << 30, ldq=1 << 37)), ({}, dict(Mq=1 << 30, ldy=1 << 37)), ({}, dict(Mk=1 << 30, ldk=1 << 37)),
    ({}, dict(Mk=1 << 30, ldv=1 << 37)), (dict(heads=1 << 20, kv_heads=1, q_head_stride=1 << 37), {}),
    (dict(heads=1 << 20, kv_heads=1, y_head_stride=1 << 37), {}), (dict(heads=1 << 20, kv_heads=1 << 20, k_head_stride=1 << 37), {}),
    (dict(heads=1 << 20, kv_heads=1 << 20, v_head_stride=1 << 37), {}),
])
def test_attention_buffers_beyond_any_address_space(fields, args):
    """(their lengths in bytes do not fit 64 bits, where an overlap could go unseen)"""
    assert _call(_attn(**fields), **args) == B.DP_ERR_SHAPE


@pytest.mark.parametrize("kw", [dict(ldx=1 << 60), dict(ldo=1 << 60)])
def test_group_norm_buffers_beyond_any_address_space(kw):
    assert _gn(False, **kw) == B.DP_ERR_SHAPE and _gn(True, **kw) == B.DP_ERR_SHAPE


def test_attention_nothing_to_do():
    assert _call(None) == B.DP_ERR_INVALID_ARG
    assert _call(_attn(n_seq=0), q=None, k=None, v=None, y=None) == B.DP_OK
    assert _call(_attn(max_q=0)) == B.DP_OK
    assert _call(_attn(max_q=0), Mq=0) == B.DP_OK


def test_attention_takes_its_own_structure_only():
    for bad in (B.dp_weight(), 0, None):
        with pytest.raises(C.ArgumentError):
            B.dp_attention(bad, None, 64, 0, None, 64, None, 64, 0, None, 64)


GN = dict(x=A, n=2, rows=10, C_=64, ldx=64, G=8, gamma=None, beta=None, eps=1e-5, act=0, out=2 * A, ldo=64, ws=3 * A, wsb=1 << 16)


def _gn(codes, **kw):
    f = dict(GN, s_a=4 * A)
    f.update(kw)
    head = (f["x"], f["n"], f["rows"], f["C_"], f["ldx"], f["G"], f["gamma"], f["beta"], f["eps"], f["act"], f["out"], f["ldo"])
    L = B.lib()
    return (L.dp_group_norm_daq(*head, f["s_a"], f["ws"], f["wsb"], None) if codes else
            L.dp_group_norm(*head, f["ws"], f["wsb"], None))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("want,kw", [
    (B.DP_ERR_SHAPE, dict(n=-1)), (B.DP_ERR_SHAPE, dict(rows=-1)), (B.DP_ERR_SHAPE, dict(C_=60)), (B.DP_ERR_SHAPE, dict(C_=4616)),
    (B.DP_ERR_SHAPE, dict(G=0)), (B.DP_ERR_SHAPE, dict(G=5)), (B.DP_ERR_SHAPE, dict(C_=4608, G=2304, ldx=4608, ldo=4608)),
    (B.DP_ERR_SHAPE, dict(rows=(1 << 30) + 1)), (B.DP_ERR_SHAPE, dict(ldx=56)), (B.DP_ERR_SHAPE, dict(ldo=56)),
    (B.DP_ERR_SHAPE, dict(n=(1 << 23) + 1, rows=1)),
    (B.DP_ERR_INVALID_ARG, dict(gamma=A)), (B.DP_ERR_INVALID_ARG, dict(beta=A)), (B.DP_ERR_INVALID_ARG, dict(eps=-1.0)),
    (B.DP_ERR_INVALID_ARG, dict(eps=float("nan"))), (B.DP_ERR_INVALID_ARG, dict(act=2)), (B.DP_ERR_INVALID_ARG, dict(x=None)),
    (B.DP_ERR_INVALID_ARG, dict(out=None)), (B.DP_ERR_INVALID_ARG, dict(out=A)), (B.DP_ERR_INVALID_ARG, dict(out=A + 256)),
    (B.DP_ERR_ALIGN, dict(x=A + 8)), (B.DP_ERR_ALIGN, dict(ldx=68)), (B.DP_ERR_ALIGN, dict(ldo=68)),
    (B.DP_ERR_ALIGN, dict(gamma=A + 2, beta=A)), (B.DP_ERR_WORKSPACE, dict(ws=None)), (B.DP_ERR_WORKSPACE, dict(ws=3 * A + 16)),
    (B.DP_ERR_WORKSPACE, dict(wsb=64)),
])
def test_group_norm_refusals(want, kw, codes):
    assert _gn(codes, **kw) == want
    assert B.lib().dp_last_error()


def test_group_norm_nothing_to_do_and_codes_need_scales():
    assert _gn(False, n=0) == B.DP_OK and _gn(True, rows=0, x=None) == B.DP_OK
    assert _gn(True, s_a=None) == B.DP_ERR_INVALID_ARG
    assert _gn(True, s_a=4 * A + 2) == B.DP_ERR_ALIGN
    assert B.dp_group_norm_workspace(2, 10, 64, 8) >= 256 and B.dp_group_norm_workspace(0, 0, 64, 8) >= 256


@pytest.mark.parametrize("kw", [dict(out=A + 96), dict(out=A + 128 * 2 + 240), dict(out=A + 16, ldx=256), dict(out=A + 256, ldx=256, ldo=512)])
def test_group_norm_columns_that_meet(kw):
    """Rows of one buffer: x's 64 columns and the output's reach each other, or do not have the same pitch."""
    assert _gn(False, **dict(dict(ldx=128, ldo=128), **kw)) == B.DP_ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [2.1e38, 2.5e38, 3.0e38])
def test_attention_scales_whose_multiple_by_log2e_is_infinite(scale):
    """(a score of 0 would be NaN)"""
    assert _call(_attn(scale=scale)) == B.DP_ERR_INVALID_ARG


@pytest.mark.parametrize("codes", [False, True])
def test_group_norm_eps_has_to_be_finite(codes):
    assert _gn(codes, eps=float("inf")) == B.DP_ERR_INVALID_ARG


@pytest.mark.parametrize("y", [A + 64 * 2, A + 128 * 2 + 16, A + 256 * 2 + 64 * 2, A + (19 * 1024 + 3 * 256 + 32) * 2])
def test_attention_heads_of_one_buffer_that_meet(y):
    """Rows of 4 heads x 4 vectors of 64: q, k, v and y alternate. y on k's vectors, reaching from v's into its own, on another head's k, and
    in the last vector of q."""
    kw = dict(ldq=1024, ldk=1024, ldv=1024, ldy=1024, Mk=20, k=A + 128, v=A + 256)
    f = dict(kv_heads=4, n_seq=1, max_k=20, **{n + "_head_stride": 256 for n in "qkvy"})
    assert _call(_attn(**f), y=y, **kw) == B.DP_ERR_INVALID_ARG
    assert _call(_attn(**f), y=A + 192 * 2, **dict(kw, q=A + 2)) == B.DP_ERR_ALIGN  # (a place of its own: the next check speaks)
