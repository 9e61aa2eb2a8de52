"""CPU checks of the calls around the attention (head norms with rotation, page
tables, paged decoding): exported as declared, sized as documented, and bad
arguments refused before anything reaches the device (fake addresses, never
dereferenced), in the library and in the binding."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2512_22234_amd as bd
from paper_2512_22234_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, SZ = 1 << 40, 1 << 36
vp = ctypes.c_void_p


def _strides(*s):
    return (ctypes.c_int64 * len(s))(*s) if s and s[0] is not None else None


def test_library_exports_every_call_of_the_header():
    text = open(os.path.join(ROOT, "include", "bd_attn.h")).read()
    names = set(re.findall(r"^(?:int|size_t|const char\*)\s+(bd_\w+)\s*\(", text, re.M))
    assert {"bd_rope_table", "bd_qk_norm_rope_fwd", "bd_qk_norm_rope_bwd", "bd_qk_norm_rope_paged", "bd_paged_plan",
            "bd_attn_paged_decode_fwd"} <= names
    for n in names:
        assert hasattr(_lib.lib(), n) and getattr(_lib.lib(), n).argtypes is not None, n


# Two tokens x (2 + 1 + 1) heads of 64 as one fused projection.
FUSED = (2 * 256, 256, 64) * 3


def _rope_args(a):
    return (vp(a["wq"]), vp(a["wk"]), vp(a["rope"]), a["n_rope"], vp(a["pos"]), a["pos_stride"])


def _rope_base(**kw):
    a = dict(Q=A, K=A + 256, V=A + 384, st=FUSED, wq=A + SZ, wk=A + 2 * SZ, rope=A + 3 * SZ, n_rope=10, pos=A + 4 * SZ,
             pos_stride=2, B=2, N=2, Hq=2, Hkv=1, D=64, eps=1e-6, dtype=0, wdtype=0, qo=A + 5 * SZ, ko=A + 6 * SZ,
             vo=A + 7 * SZ)
    a.update(kw)
    return a


def _rope_fwd(**kw):
    a = _rope_base(**kw)
    return _lib.lib().bd_qk_norm_rope_fwd(vp(a["Q"]), vp(a["K"]), vp(a["V"]), _strides(*a["st"]), *_rope_args(a), a["B"],
                                          a["N"], a["Hq"], a["Hkv"], a["D"], a["eps"], a["dtype"], a["wdtype"],
                                          vp(a["qo"]), vp(a["ko"]), vp(a["vo"]), None)


ROPE_REFUSALS = [
    (dict(D=96), 2), (dict(D=256), 2), (dict(dtype=3), 2), (dict(wdtype=2), 2), (dict(dtype=1, wdtype=0), 2),
    (dict(B=-1), 1), (dict(N=-1), 1), (dict(B=1 << 15, N=1 << 14), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1),
    (dict(Hq=(1 << 14) + 1), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(n_rope=0), 1), (dict(pos_stride=-1), 1),
    (dict(Q=0), 1), (dict(wk=0), 1), (dict(rope=0), 1), (dict(pos=0), 1), (dict(st=(None,)), 1),
    (dict(Q=A + 8), 1), (dict(wq=A + SZ + 8), 1), (dict(pos=A + 4 * SZ + 2), 1),
    (dict(st=(512, 252, 64) * 3), 1), (dict(st=(512, -256, 64) * 3), 1), (dict(st=(1 << 50, 256, 64) * 3), 1),
]


@pytest.mark.parametrize("kw,status", ROPE_REFUSALS + [
    (dict(qo=0), 1), (dict(vo=A + 7 * SZ + 8), 1),
    (dict(ko=A + 256), 1),                     # an output inside the projection
    (dict(ko=A + 5 * SZ + 512), 1),            # ... inside another output
    (dict(vo=A + 3 * SZ + 256), 1),            # ... inside the table
])
def test_norm_rope_refusals(kw, status):
    assert _rope_fwd(**kw) == status


def test_norm_rope_without_tokens_enqueues_nothing():
    assert _rope_fwd(B=0, Q=0, K=0, V=0) == 0 and _rope_fwd(N=0, qo=0) == 0


def _rope_bwd(**kw):
    a = _rope_base(gst=FUSED, dqo=A + 8 * SZ, dko=A + 9 * SZ, dvo=A + 10 * SZ, dq=A + 11 * SZ, dk=A + 11 * SZ + 256,
                   dv=A + 11 * SZ + 384, dwq=A + 12 * SZ, dwk=A + 13 * SZ, ws=A + 14 * SZ, ws_bytes=1 << 20)
    a.update(kw)
    return _lib.lib().bd_qk_norm_rope_bwd(vp(a["dqo"]), vp(a["dko"]), vp(a["dvo"]), vp(a["Q"]), vp(a["K"]),
                                          _strides(*a["st"]), *_rope_args(a), a["B"], a["N"], a["Hq"], a["Hkv"], a["D"],
                                          a["eps"], a["dtype"], a["wdtype"], vp(a["dq"]), vp(a["dk"]), vp(a["dv"]),
                                          _strides(*a["gst"]), vp(a["dwq"]), vp(a["dwk"]), vp(a["ws"]), a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", ROPE_REFUSALS + [
    (dict(dwq=0), 1), (dict(dwk=A + 12 * SZ), 1), (dict(dqo=0), 1), (dict(dv=0), 1), (dict(gst=(None,)), 1), (dict(ws=0), 1),
    (dict(ws_bytes=64), 3),
    (dict(gst=(512, 0, 64) * 3), 1),           # two tokens' gradients in one place
    (dict(gst=(256, 256, 64) * 3), 1),         # ... two sequences'
    (dict(gst=(512, 256, 32) * 3), 1),         # ... two heads'
    (dict(dk=A + 11 * SZ + 128), 1),           # keys' gradients among the queries'
    (dict(dv=A + 11 * SZ + 512), 1),           # values' in the next token's
    (dict(dq=A + 256), 1), (dict(ws=A + 8 * SZ), 1), (dict(dwk=A + 14 * SZ), 1),
])
def test_norm_rope_backward_refusals(kw, status):
    assert _rope_bwd(**kw) == status


def test_norm_rope_workspace_bytes():
    f = bd.bd_qk_norm_rope_workspace_bytes
    # D float32 sums for every workgroup's tokens (32 or 64 a workgroup) and heads of a kind (one here)
    assert f(1, 33, 3, 2, 128) == 2 * (3 + 2) * 128 * 4
    assert f(1, 64, 1, 1, 64, 1) == 2 * 64 * 4
    assert f(0, 5, 1, 1, 64) == f(3, 0, 1, 1, 64) == 0
    for bad in [(1, 4, 0, 1, 64), (1, 4, 1, 1, 96), (1 << 15, 1 << 14, 1, 1, 64), (1, 4, 1, 1, 64, 5), (-1, 4, 1, 1, 64)]:
        assert f(*bad) == 0, bad


def _rope_paged(**kw):
    a = _rope_base(slots=A + 8 * SZ, kp=A + 9 * SZ, vp=A + 10 * SZ, num=8, P=16, sp=1024, sh=1024, sr=64)
    a.update(kw)
    return _lib.lib().bd_qk_norm_rope_paged(vp(a["Q"]), vp(a["K"]), vp(a["V"]), _strides(*a["st"]), *_rope_args(a),
                                            vp(a["slots"]), a["B"], a["N"], a["Hq"], a["Hkv"], a["D"], a["eps"],
                                            a["dtype"], a["wdtype"], vp(a["qo"]), vp(a["kp"]), vp(a["vp"]), a["num"],
                                            a["P"], a["sp"], a["sh"], a["sr"], None)


@pytest.mark.parametrize("kw,status", ROPE_REFUSALS + [
    (dict(dtype=1, wdtype=1), 2),              # float32 rows have no pages
    (dict(P=24), 1), (dict(P=8), 1), (dict(P=1 << 16), 1), (dict(P=0), 1), (dict(num=0), 1), (dict(num=1 << 28), 1),
    (dict(kp=0), 1), (dict(vp=A + 10 * SZ + 8), 1), (dict(slots=0), 1), (dict(slots=A + 8 * SZ + 2), 1), (dict(qo=0), 1),
    (dict(sr=32), 1), (dict(sp=512), 1), (dict(Hkv=2, sh=512, sp=2048), 1), (dict(sr=60), 1), (dict(sp=-1024), 1),
    (dict(vp=A + 9 * SZ + 1024), 1),           # the values' pages are the next keys'
    (dict(vp=A + 9 * SZ), 1),
    (dict(kp=A + 5 * SZ), 1), (dict(vp=A + 3 * SZ), 1), (dict(qo=A + 9 * SZ + 64), 1),
])
def test_norm_rope_paged_refusals(kw, status):
    assert _rope_paged(**kw) == status


def test_interleaved_pages_are_apart():
    """K and V of one array [pages, 2, ...]: accepted up to the next check (here: a missing pointer)."""
    ok = dict(vp=A + 9 * SZ + 2048, sp=2048, qo=0, B=0)
    assert _rope_paged(**ok) == 0
    assert _rope_paged(**dict(ok, vp=A + 9 * SZ + 1024)) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), 1), (dict(n=(1 << 25) + 1), 1), (dict(D=32), 2), (dict(f=0), 1), (dict(t=0), 1), (dict(f=A + 4), 1),
    (dict(t=A + SZ + 8), 1), (dict(t=A + 16), 1),
])
def test_rope_table_refusals(kw, status):
    a = dict(f=A, n=4, D=64, t=A + SZ)
    a.update(kw)
    assert _lib.lib().bd_rope_table(vp(a["f"]), a["n"], a["D"], vp(a["t"]), None) == status


def _plan(**kw):
    a = dict(old=A, new=A + SZ, table=A + 2 * SZ, B=3, width=4, ts=4, free=A + 3 * SZ, n_free=10, head=A + 4 * SZ, num=20,
             P=16, S=4, total=0, lens=A + 5 * SZ, cu=A + 6 * SZ, slots=A + 7 * SZ, pos=A + 8 * SZ, state=A + 9 * SZ)
    a.update(kw)
    return _lib.lib().bd_paged_plan(vp(a["old"]), vp(a["new"]), vp(a["table"]), a["B"], a["width"], a["ts"], vp(a["free"]),
                                    a["n_free"], vp(a["head"]), a["num"], a["P"], a["S"], a["total"], vp(a["lens"]),
                                    vp(a["cu"]), vp(a["slots"]), vp(a["pos"]), vp(a["state"]), None)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(B=(1 << 16) + 1), dict(width=0), dict(ts=3), dict(P=20), dict(P=8), dict(width=1 << 27, ts=1 << 27),
    dict(num=0), dict(num=1 << 28), dict(n_free=-1), dict(S=-1), dict(S=1 << 29), dict(S=0, total=-1),
    dict(S=0, total=(1 << 30) + 1), dict(old=0), dict(new=0), dict(table=0), dict(free=0), dict(head=0), dict(lens=0),
    dict(cu=0), dict(slots=0), dict(pos=0), dict(state=0), dict(old=A + 2), dict(slots=A + 7 * SZ + 1),
    dict(lens=A + 4),                          # the new lengths over the old ones
    dict(state=A + 4 * SZ), dict(cu=A + 5 * SZ + 8), dict(table=A + 3 * SZ + 8), dict(pos=A + 7 * SZ + 16),
])
def test_paged_plan_refusals(kw):
    assert _plan(**kw) == 1


def test_paged_decode_workspace_bytes():
    f = bd.bd_attn_paged_decode_workspace_bytes
    assert f(64, 4, 32, 8, 128, 64, 128) == bd.bd_attn_decode_workspace_bytes(64, 4, 32, 8, 128, 8192) > 0
    for bad in [(2, 1, 4, 2, 64, 24, 8), (2, 1, 4, 2, 64, 16, 0), (2, 1, 4, 2, 64, 16, (1 << 18) + 1), (2, 0, 4, 2, 64, 16, 8),
                (2, 1, 3, 2, 64, 16, 8), (2, 1, 4, 2, 96, 16, 8), (2, 1, 4, 2, 64, 16, 8, 1), (0, 1, 4, 2, 64, 16, 8),
                (1 << 12, 1 << 10, 32, 32, 64, 16, 8)]:
        assert f(*bad) == 0, bad


def _paged(**kw):
    a = dict(Q=A, kp=A + SZ, vp=A + 2 * SZ, table=A + 3 * SZ, lens=A + 4 * SZ, kn=A + 5 * SZ, vn=A + 6 * SZ, B=2, S=4, Hq=2,
             Hkv=1, D=64, num=8, P=16, width=4, ts=4, sp=1024, sh=1024, sr=64, scale=0.0, dtype=0, O=A + 7 * SZ,
             lse=A + 8 * SZ, ws=A + 9 * SZ, ws_bytes=1 << 30)
    a.update(kw)
    return _lib.lib().bd_attn_paged_decode_fwd(
        vp(a["Q"]), vp(a["kp"]), vp(a["vp"]), vp(a["table"]), vp(a["lens"]), vp(a["kn"]), vp(a["vn"]), a["B"], a["S"],
        a["Hq"], a["Hkv"], a["D"], a["num"], a["P"], a["width"], a["ts"], a["sp"], a["sh"], a["sr"], a["scale"],
        a["dtype"], vp(a["O"]), vp(a["lse"]), vp(a["ws"]), a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(D=96), 2), (dict(dtype=1), 2), (dict(Hq=3, Hkv=2), 1), (dict(B=0), 1), (dict(S=0), 1),
    (dict(P=48), 1), (dict(P=8), 1), (dict(width=0), 1), (dict(width=1 << 19, ts=1 << 19), 1), (dict(num=0), 1),
    (dict(num=1 << 27), 1), (dict(ts=3), 1), (dict(ts=-1), 1), (dict(sp=12), 1), (dict(sr=32), 1), (dict(sr=(1 << 20) + 8), 1),
    (dict(sp=1 << 31), 1), (dict(P=1 << 12, sr=(1 << 18) + 8), 1),
    (dict(sh=-8), 1), (dict(scale=float("nan")), 1),
    (dict(Q=0), 1), (dict(kp=0), 1), (dict(vp=0), 1), (dict(table=0), 1), (dict(lens=0), 1), (dict(kn=0), 1),
    (dict(vn=0), 1), (dict(O=0), 1), (dict(lse=0), 1), (dict(ws=0), 1),
    (dict(Q=A + 8), 1), (dict(kp=A + SZ + 8), 1), (dict(table=A + 3 * SZ + 2), 1), (dict(ws=A + 9 * SZ + 8), 1),
    (dict(ws_bytes=64), 3),
    (dict(O=A + 64), 1), (dict(O=A + SZ + 4096), 1), (dict(lse=A + 3 * SZ), 1), (dict(ws=A + 7 * SZ + 256), 1),
])
def test_paged_decode_refusals(kw, status):
    assert _paged(**kw) == status


# The binding's own checks (tensors on the CPU are refused before a pointer leaves it only for shape,
# type and layout; these calls all fail there).

def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("change,error", [
    (dict(q=_t(2, 3, 4, 64, dtype=torch.float16)), TypeError), (dict(k=_t(2, 3, 2, 64, dtype=torch.float32)), TypeError),
    (dict(k=_t(3, 3, 2, 64)), ValueError), (dict(v=_t(2, 3, 1, 64)), ValueError), (dict(q=_t(4, 64)), ValueError),
    (dict(wq=_t(64, dtype=torch.float16)), TypeError), (dict(wk=_t(32)), ValueError), (dict(wk=_t(64, dtype=torch.float32)), TypeError),
    (dict(rope=_t(9, 32, dtype=torch.float32)), ValueError), (dict(rope=_t(9, 64)), TypeError),
    (dict(pos=_i(2, 4)), ValueError), (dict(pos=torch.zeros(2, 3, dtype=torch.int64)), TypeError), (dict(pos=_i(2)), ValueError),
    (dict(q=_t(2, 3, 4, 128)[..., ::2]), ValueError), (dict(q=_t(2, 3, 4, 68)[..., :64]), ValueError),
])
def test_norm_rope_binding_refusals(change, error):
    a = dict(q=_t(2, 3, 4, 64), k=_t(2, 3, 2, 64), v=_t(2, 3, 2, 64), wq=_t(64), wk=_t(64), rope=_t(9, 64, dtype=torch.float32),
             pos=_i(2, 3))
    a.update(change)
    with pytest.raises(error):
        bd.bd_qk_norm_rope_fwd(*a.values())
    with pytest.raises(error):
        bd.bd_qk_norm_rope_paged(*a.values(), _i(2, 3), _t(5, 2, 16, 64), _t(5, 2, 16, 64))


@pytest.mark.parametrize("change,error", [
    (dict(slots=_i(6)), ValueError), (dict(kp=_t(5, 3, 16, 64)), ValueError), (dict(vp=_t(4, 2, 16, 64)), ValueError),
    (dict(vp=_t(5, 2, 16, 64, dtype=torch.float32)), TypeError), (dict(kp=_t(5, 2, 16, 128)[..., ::2]), ValueError),
    (dict(kp=_t(5, 16, 2, 64).permute(0, 2, 1, 3)), ValueError), (dict(kp=_t(2, 16, 64)), ValueError),
])
def test_pages_binding_refusals(change, error):
    a = dict(slots=_i(2, 3), kp=_t(5, 2, 16, 64), vp=_t(5, 2, 16, 64))
    a.update(change)
    with pytest.raises(error):
        bd.bd_qk_norm_rope_paged(_t(2, 3, 4, 64), _t(2, 3, 2, 64), _t(2, 3, 2, 64), _t(64), _t(64),
                                 _t(9, 64, dtype=torch.float32), _i(2, 3), *a.values())
    if "slots" not in change:
        with pytest.raises((ValueError, TypeError)):
            bd.bd_attn_paged_decode_fwd(_t(2, 4, 1, 64), a["kp"], a["vp"], _i(2, 3), _i(2))


@pytest.mark.parametrize("change,error", [
    (dict(q=_t(2, 4, 1, 64, dtype=torch.float32)), TypeError),
    (dict(table=_i(3, 3)), ValueError), (dict(table=torch.zeros(2, 3, dtype=torch.int64)), TypeError), (dict(table=_i(2, 6)[:, ::2]), ValueError),
    (dict(lens=_i(3)), ValueError), (dict(kn=_t(2, 2, 1, 64)), ValueError), (dict(kn=_t(2, 2, 2, 64), vn=_t(2, 2, 2, 64)), ValueError),
    (dict(q=_t(2, 4, 2, 128)[..., :64]), ValueError),
])
def test_paged_decode_binding_refusals(change, error):
    a = dict(q=_t(2, 4, 1, 64), kp=_t(5, 2, 16, 64), vp=_t(5, 2, 16, 64), table=_i(2, 3), lens=_i(2), kn=None, vn=None)
    a.update(change)
    with pytest.raises(error):
        bd.bd_attn_paged_decode_fwd(*a.values())


@pytest.mark.parametrize("change,kw,error", [
    (dict(new=_i(3)), dict(S=4), ValueError), (dict(table=_i(3, 4)), dict(S=4), ValueError), (dict(old=_i(2, 1)), dict(S=4), ValueError),
    (dict(table=torch.zeros(2, 4, dtype=torch.int64)), dict(S=4), TypeError), (dict(table=_i(2, 8)[:, ::2]), dict(S=4), ValueError),
    (dict(head=_i(2)), dict(S=4), ValueError), (dict(free=_i(2, 2)), dict(S=4), ValueError), ({}, {}, ValueError), ({}, dict(S=0), ValueError),
    (dict(free=torch.zeros(4, dtype=torch.int64)), dict(total=4), TypeError), ({}, dict(S=4, slots=_i(8)), ValueError),
])
def test_paged_plan_binding_refusals(change, kw, error):
    a = dict(old=_i(2), new=_i(2), table=_i(2, 4), free=_i(8), head=_i(1))
    a.update(change)
    with pytest.raises(error):
        bd.bd_paged_plan(*a.values(), 16, 16, **kw)


# Strides whose products wrap 64 bits to nothing, so that the spans would seem to fit.
WRAPS = (0, 1 << 40, 64) * 3


def test_strides_past_any_memory_are_refused():
    rows = dict(B=1, N=(1 << 24) + 1, pos_stride=0)
    assert _rope_fwd(**rows, st=WRAPS) == 1
    assert _rope_bwd(**rows, st=WRAPS) == 1
    assert _rope_bwd(**rows, gst=WRAPS, ws_bytes=1 << 34) == 1
    assert _rope_paged(**rows, st=WRAPS) == 1
    seqs = dict(B=(1 << 14) + 1, pos_stride=1 << 48)
    assert _rope_fwd(**seqs) == 1 and _rope_bwd(**seqs, ws_bytes=1 << 30) == 1 and _rope_paged(**seqs) == 1
    assert _rope_paged(num=(1 << 24) + 1, sp=1 << 40) == 1
    assert _plan(B=(1 << 14) + 1, ts=1 << 48) == 1
    assert _paged(B=(1 << 14) + 1, ts=1 << 48, ws_bytes=1 << 40) == 1


E = A + 11 * SZ  # the queries' gradient


@pytest.mark.parametrize("kw", [
    # one head of 64, the keys' gradient 64 behind the queries' in every token: two sequences a token and a half apart,
    dict(gst=(192, 128, 64) * 3, dv=A + 15 * SZ),
    # ... and less than a sequence's span apart, which puts (1, 0) of one on (0, 9) of the other
    dict(N=10, gst=(9064, 1000, 64) * 3, dv=A + 15 * SZ),
    dict(B=10, gst=(1000, 9064, 64) * 3, dv=A + 15 * SZ),
    # the values' gradient, behind both
    dict(gst=(256, 192, 64, 256, 192, 64, 256, 192, 64), dk=A + 15 * SZ, dv=E + 128),
])
def test_interleaved_gradients_that_meet_are_refused(kw):
    a = dict(Hq=1, Hkv=1, dq=E, dk=E + 128, pos_stride=0)
    a.update(kw)
    assert _rope_bwd(**a) == 1


def _fused_call(Hq, Hkv, qkv=_t(2, 3, 8 * 64)):
    bd.qkv_norm_rope(qkv, Hq, Hkv, _t(64), _t(64), _t(9, 64, dtype=torch.float32), _i(2, 3))


def test_fused_heads_are_taken_at_their_present_value():
    """A scalar that changed between two calls is checked again (the first call gets as far as the device)."""
    for Hq, change in ((torch.tensor(6), lambda x: x.fill_(60)), (np.array(6), lambda x: x.fill(60))):
        for _ in range(2):
            with pytest.raises(Exception) as e:
                _fused_call(Hq, 1)
            assert "heads" not in str(e.value)
        change(Hq)
        with pytest.raises(ValueError, match="60/1 heads"):
            _fused_call(Hq, 1)
    with pytest.raises(TypeError):
        _fused_call(6.0, 1)


@pytest.mark.parametrize("change,kw", [
    ({}, dict(S=4, page_size=(1 << 32) + 16)), ({}, dict(S=4, num_pages=(1 << 32) + 16)), ({}, dict(S=4, num_pages=16 - (1 << 32))),
    ({}, dict(total=(1 << 32) + 8, slots=_i(1).expand((1 << 32) + 8))), ({}, dict(S=(1 << 32) + 4, slots=_i(1, 1).expand(2, (1 << 32) + 4))),
    (dict(table=torch.empty((2, (1 << 32) + 4), dtype=torch.int32, device="meta")), dict(S=4)),
    (dict(free=torch.empty((1 << 32) + 4, dtype=torch.int32, device="meta")), dict(S=4)),
])
def test_paged_plan_sizes_past_32_bits_are_refused(change, kw):
    """They reach the library as C ints, where they would count as what is left of them."""
    a = dict(old=_i(2), new=_i(2), table=_i(2, 4), free=_i(8), head=_i(1))
    if change:
        a = {n: t.to("meta") for n, t in a.items()}
    a.update(change)
    kw = dict(dict(num_pages=16, page_size=16), **kw)
    with pytest.raises(ValueError, match="32 bits"):
        bd.bd_paged_plan(*a.values(), **kw)


def test_other_sizes_past_32_bits_are_refused():
    big = 1 << 32
    with pytest.raises(ValueError, match="32 bits"):
        bd.bd_rope_table(big + 4, 64, device="cpu")
    with pytest.raises(ValueError, match="32 bits"):
        bd.bd_rope_table(4, big + 64, device="cpu")
    pages = _t(1, 2, 16, 64).expand(big + 5, 2, 16, 64)
    with pytest.raises(ValueError, match="32 bits"):
        bd.bd_attn_paged_decode_fwd(_t(2, 4, 1, 64), pages, pages, _i(2, 3), _i(2))
    q, pages, lens, table = (torch.empty(x, dtype=t, device="meta") for x, t in (
        ((2, 4, 1, 64), torch.bfloat16), ((5, 2, 16, 64), torch.bfloat16), ((2,), torch.int32), ((2, big + 3), torch.int32)))
    with pytest.raises(ValueError, match="32 bits"):
        bd.bd_attn_paged_decode_fwd(q, pages, pages, table, lens)
    for i in range(7):
        sizes = [2, 1, 4, 2, 64, 16, 8]
        sizes[i] += big
        assert bd.bd_attn_paged_decode_workspace_bytes(*sizes) == 0
    for i in range(5):
        sizes = [1, 33, 3, 2, 128]
        sizes[i] += big
        assert bd.bd_qk_norm_rope_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("k,v", [
    (_t(1, 2, 16, 64), _t(1, 2, 2, 16, 64)[:, 0]),                          # one page
    (_t(5, 1, 16, 64), _t(5, 16, 1, 64).permute(0, 2, 1, 3)),               # one head
])
def test_pages_alike_but_for_strides_without_a_step(k, v):
    """A dimension of one has no stride of its own: such K and V pages lie alike (the call gets as far as the device)."""
    with pytest.raises(Exception) as e:
        bd.bd_attn_paged_decode_fwd(_t(2, 4, 1, 64), k, v, _i(2, 3), _i(2))
    assert "strides" not in str(e.value)


@pytest.mark.parametrize("ws", [torch.empty(1 << 28, dtype=torch.uint8, device="meta"),
                                torch.empty((1 << 28, 2), dtype=torch.uint8, device="meta")[:, 0]])
def test_workspace_elsewhere_or_with_gaps_is_refused(ws):
    dev = "cpu" if ws.is_contiguous() else "meta"
    q, pages, lens, table = (torch.empty(x, dtype=t, device=dev) for x, t in (
        ((2, 4, 1, 64), torch.bfloat16), ((5, 2, 16, 64), torch.bfloat16), ((2,), torch.int32), ((2, 3), torch.int32)))
    with pytest.raises(ValueError, match="workspace"):
        bd.bd_attn_paged_decode_fwd(q, pages, pages, table, lens, workspace=ws)
