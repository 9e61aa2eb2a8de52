"""CPU checks of decoding with shared prefixes, page summaries, the choice of pages and
decoding over lists: exported as declared, sized as documented, and bad arguments
refused before anything reaches the device (fake addresses, never dereferenced), in
the library and in the binding."""
import ctypes

import pytest
import torch

import paper_2512_22234_amd as bd
from paper_2512_22234_amd import _lib

A, SZ = 1 << 40, 1 << 36
vp = ctypes.c_void_p
BIG = (1 << 31) - 1


def _shared(**kw):
    a = dict(Q=A, kp=A + SZ, vp=A + 2 * SZ, sizes=A + 11 * SZ, groups=2, pt=A + 12 * SZ, pw=3, ps=3, pl=A + 13 * SZ,
             table=A + 3 * SZ, lens=A + 4 * SZ, kn=A + 5 * SZ, vn=A + 6 * SZ, B=4, S=4, Hq=4, Hkv=2, D=64, num=9, P=16, width=5,
             ts=5, sp=2048, sh=1024, sr=64, scale=0.0, dtype=0, O=A + 7 * SZ, lse=A + 8 * SZ, ws=A + 9 * SZ, ws_bytes=1 << 28)
    a.update(kw)
    p = lambda n: vp(a[n])  # noqa: E731
    return _lib.lib().bd_attn_paged_shared_decode_fwd(
        p("Q"), p("kp"), p("vp"), p("sizes"), a["groups"], p("pt"), a["pw"], a["ps"], p("pl"), p("table"), p("lens"), p("kn"),
        p("vn"), a["B"], a["S"], a["Hq"], a["Hkv"], a["D"], a["num"], a["P"], a["width"], a["ts"], a["sp"], a["sh"], a["sr"],
        a["scale"], a["dtype"], p("O"), p("lse"), p("ws"), a["ws_bytes"], None)


PAGED_REFUSALS = [
    (dict(D=96), 2), (dict(dtype=1), 2), (dict(B=0), 1), (dict(S=0), 1), (dict(Hq=5), 1), (dict(Hkv=0), 1), (dict(Hq=-4, Hkv=-2), 1),
    (dict(P=24), 1), (dict(P=8), 1), (dict(num=0), 1), (dict(width=0), 1), (dict(width=1 << 19), 1), (dict(num=1 << 28), 1),
    (dict(sr=72 * 8 + 4), 1), (dict(sr=32), 1), (dict(sp=-8), 1), (dict(sp=1 << 31), 1), (dict(sh=12), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(Q=0), 1), (dict(kp=0), 1), (dict(vp=0), 1), (dict(table=0), 1), (dict(lens=0), 1), (dict(kn=0), 1), (dict(vn=0), 1),
    (dict(O=0), 1), (dict(lse=0), 1), (dict(ws=0), 1),
    (dict(Q=A + 8), 1), (dict(table=A + 3 * SZ + 2), 1), (dict(lens=A + 4 * SZ + 1), 1), (dict(O=A + 7 * SZ + 8), 1),
    (dict(ws=A + 9 * SZ + 8), 1), (dict(ws_bytes=64), 3),
    (dict(O=A + 64), 1), (dict(O=A + SZ + 4096), 1), (dict(lse=A + 3 * SZ), 1), (dict(ws=A + 7 * SZ + 256), 1),
    (dict(B=1 << 22, S=1 << 4), 1),
]


@pytest.mark.parametrize("kw,status", PAGED_REFUSALS + [
    (dict(groups=0), 1), (dict(groups=-1), 1), (dict(groups=(1 << 16) + 1), 1), (dict(pw=0), 1), (dict(pw=1 << 19), 1), (dict(ps=-3), 1),
    (dict(ps=2), 1), (dict(ts=4), 1), (dict(sizes=0), 1), (dict(pt=0), 1), (dict(pl=0), 1), (dict(sizes=A + 11 * SZ + 2), 1),
    (dict(pt=A + 12 * SZ + 1), 1), (dict(pl=A + 13 * SZ + 3), 1),
    (dict(O=A + 11 * SZ), 1), (dict(lse=A + 12 * SZ + 4), 1), (dict(ws=A + 13 * SZ), 1),   # outputs on the groups' arrays
    (dict(groups=1 << 16, ps=1 << 48, pw=3), 1), (dict(B=(1 << 14) + 1, ts=1 << 48, ws_bytes=1 << 40), 1),
    (dict(B=1 << 16, groups=1 << 16, pw=1 << 18, ps=1 << 18), 1),                          # more tiles than 31 bits count
])
def test_shared_decode_refusals(kw, status):
    assert _shared(**kw) == status


def _sparse(**kw):
    a = dict(Q=A, kp=A + SZ, vp=A + 2 * SZ, table=A + 3 * SZ, lens=A + 4 * SZ, kn=A + 5 * SZ, vn=A + 6 * SZ, B=4, S=4, Hq=4, Hkv=2,
             D=64, num=9, P=16, width=5, sp=2048, sh=1024, sr=64, scale=0.0, dtype=0, O=A + 7 * SZ, lse=A + 8 * SZ, ws=A + 9 * SZ,
             ws_bytes=1 << 28)
    a.update(kw)
    p = lambda n: vp(a[n])  # noqa: E731
    return _lib.lib().bd_attn_paged_sparse_decode_fwd(
        p("Q"), p("kp"), p("vp"), p("table"), p("lens"), p("kn"), p("vn"), a["B"], a["S"], a["Hq"], a["Hkv"], a["D"], a["num"],
        a["P"], a["width"], a["sp"], a["sh"], a["sr"], a["scale"], a["dtype"], p("O"), p("lse"), p("ws"), a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", PAGED_REFUSALS + [(dict(lse=A + 3 * SZ + 4 * 2 * 5 * 4 - 4), 1)])  # on the last list
def test_sparse_decode_refusals(kw, status):
    assert _sparse(**kw) == status


def _summarize(**kw):
    a = dict(kp=A, table=A + SZ, before=A + 2 * SZ, lens=A + 3 * SZ, B=2, Hkv=2, D=64, num=9, P=16, width=4, ts=4, sp=2048, sh=1024,
             sr=64, dtype=0, out=A + 4 * SZ)
    a.update(kw)
    p = lambda n: vp(a[n])  # noqa: E731
    return _lib.lib().bd_paged_summarize(p("kp"), p("table"), p("before"), p("lens"), a["B"], a["Hkv"], a["D"], a["num"], a["P"],
                                         a["width"], a["ts"], a["sp"], a["sh"], a["sr"], a["dtype"], p("out"), None)


@pytest.mark.parametrize("kw,status", [
    (dict(D=96), 2), (dict(dtype=1), 2), (dict(B=0), 1), (dict(Hkv=0), 1), (dict(P=24), 1), (dict(num=0), 1), (dict(num=1 << 28), 1),
    (dict(width=0), 1), (dict(width=1 << 27), 1), (dict(ts=3), 1), (dict(ts=-4), 1), (dict(sr=60), 1), (dict(sh=-8), 1),
    (dict(sp=1 << 50), 1), (dict(B=1 << 22), 1), (dict(B=(1 << 14) + 1, ts=1 << 48), 1),
    (dict(kp=0), 1), (dict(table=0), 1), (dict(before=0), 1), (dict(lens=0), 1), (dict(out=0), 1),
    (dict(kp=A + 8), 1), (dict(table=A + SZ + 2), 1), (dict(lens=A + 3 * SZ + 1), 1), (dict(out=A + 4 * SZ + 8), 1),
    (dict(out=A + 4096), 1), (dict(out=A + SZ), 1), (dict(out=A + 2 * SZ), 1), (dict(out=A + 3 * SZ - 9 * 2 * 2 * 64 * 2 + 16), 1),
])
def test_summarize_refusals(kw, status):
    assert _summarize(**kw) == status


def _select(**kw):
    a = dict(Q=A, s=A + SZ, table=A + 2 * SZ, lens=A + 3 * SZ, B=2, S=4, Hq=4, Hkv=2, D=64, num=9, P=16, width=5, ts=5, budget=3,
             first=1, last=1, dtype=0, lists=A + 4 * SZ, keys=A + 5 * SZ, ws=A + 6 * SZ, ws_bytes=1 << 20)
    a.update(kw)
    p = lambda n: vp(a[n])  # noqa: E731
    return _lib.lib().bd_paged_select(p("Q"), p("s"), p("table"), p("lens"), a["B"], a["S"], a["Hq"], a["Hkv"], a["D"], a["num"],
                                      a["P"], a["width"], a["ts"], a["budget"], a["first"], a["last"], a["dtype"], p("lists"),
                                      p("keys"), p("ws"), a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(D=96), 2), (dict(dtype=1), 2), (dict(B=0), 1), (dict(S=0), 1), (dict(Hq=5), 1), (dict(Hkv=0), 1), (dict(P=24), 1),
    (dict(num=0), 1), (dict(num=1 << 28), 1), (dict(width=0), 1), (dict(width=1 << 19), 1), (dict(ts=4), 1), (dict(ts=-1), 1),
    (dict(budget=0), 1), (dict(budget=1 << 19), 1), (dict(first=-1), 1), (dict(last=-1), 1), (dict(first=2, last=2), 1),
    (dict(first=BIG, last=BIG), 1), (dict(B=1 << 20, width=1 << 10, ts=1 << 10, ws_bytes=1 << 40), 1), (dict(B=1 << 22), 1),
    (dict(B=1 << 24, S=4), 1), (dict(B=(1 << 14) + 1, ts=1 << 48), 1),
    (dict(Q=0), 1), (dict(s=0), 1), (dict(table=0), 1), (dict(lens=0), 1), (dict(lists=0), 1), (dict(keys=0), 1), (dict(ws=0), 1),
    (dict(Q=A + 2), 1), (dict(s=A + SZ + 8), 1), (dict(ws=A + 6 * SZ + 8), 1), (dict(lists=A + 4 * SZ + 2), 1), (dict(ws_bytes=64), 3),
    (dict(lists=A), 1), (dict(keys=A + SZ), 1), (dict(ws=A + 2 * SZ), 1), (dict(keys=A + 4 * SZ + 4), 1), (dict(ws=A + 3 * SZ), 1),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status


def test_workspace_sizes():
    """Sizes grow with what they hold, are 0 for what the calls refuse, and sizes past 32 bits never reach the library."""
    shared = bd.bd_attn_paged_shared_decode_workspace_bytes
    assert shared(4, 2, 4, 4, 2, 64, 16, 3, 5) >= bd.bd_attn_paged_decode_workspace_bytes(4, 4, 4, 2, 64, 16, 5)
    assert shared(4, 0, 4, 4, 2, 64, 16, 3, 5) == shared(4, 2, 4, 4, 2, 96, 16, 3, 5) == shared(4, 2, 4, 4, 2, 64, 24, 3, 5) == 0
    assert shared((1 << 32) + 4, 2, 4, 4, 2, 64, 16, 3, 5) == shared(4, 2, 4, 4, 2, 64, 16, (1 << 32) + 3, 5) == 0
    sparse = bd.bd_attn_paged_sparse_decode_workspace_bytes
    assert sparse(4, 4, 4, 2, 64, 16, 5) == bd.bd_attn_paged_decode_workspace_bytes(4, 4, 4, 2, 64, 16, 5)
    assert sparse(4, 4, 5, 2, 64, 16, 5) == sparse((1 << 32) + 4, 4, 4, 2, 64, 16, 5) == 0
    select = bd.bd_paged_select_workspace_bytes
    assert select(2, 4, 4, 2, 64, 16, 5, 3) >= 2 * 2 * 5 * 8
    assert select(2, 4, 4, 2, 64, 16, 5, 0) == select((1 << 32) + 2, 4, 4, 2, 64, 16, 5, 3) == 0


# The binding's own checks, on the CPU.

def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("change,error", [
    (dict(q=_t(3, 4, 1, 64, dtype=torch.float32)), TypeError), (dict(q=_t(3, 4, 64)), ValueError), (dict(kp=_t(5, 16, 64)), ValueError),
    (dict(vp=_t(5, 2, 16, 64, dtype=torch.float16)), TypeError), (dict(sizes=_i(2, 1)), ValueError), (dict(sizes=_i(3)), ValueError),
    (dict(sizes=torch.zeros(2, dtype=torch.int64)), TypeError), (dict(pt=_i(3, 4)), ValueError), (dict(pt=_i(2, 8)[:, ::2]), ValueError),
    (dict(pt=torch.zeros(2, 4, dtype=torch.int64)), TypeError), (dict(pl=_i(3)), ValueError), (dict(table=_i(2, 4)), ValueError),
    (dict(lens=_i(2)), ValueError), (dict(kn=_t(3, 2, 1, 64)), ValueError), (dict(kn=_t(3, 2, 2, 64), vn=_t(3, 2, 1, 64)), ValueError),
])
def test_shared_decode_binding_refusals(change, error):
    a = dict(q=_t(3, 4, 1, 64), kp=_t(5, 2, 16, 64), vp=_t(5, 2, 16, 64), sizes=_i(2), pt=_i(2, 4), pl=_i(2), table=_i(3, 4),
             lens=_i(3), kn=None, vn=None)
    a.update(change)
    with pytest.raises(error):
        bd.bd_attn_paged_shared_decode_fwd(*a.values())


@pytest.mark.parametrize("change,error", [
    (dict(q=_t(3, 4, 1, 64, dtype=torch.float32)), TypeError), (dict(lists=_i(3, 4)), ValueError), (dict(lists=_i(3, 3, 4)), ValueError),
    (dict(lists=_i(3, 2, 8)[..., ::2]), ValueError), (dict(lists=torch.zeros(3, 2, 4, dtype=torch.int64)), TypeError),
    (dict(lens=_i(3)), ValueError), (dict(lens=_i(2, 3)), ValueError), (dict(kn=_t(3, 2, 1, 64)), ValueError),
])
def test_sparse_decode_binding_refusals(change, error):
    a = dict(q=_t(3, 4, 1, 64), kp=_t(5, 2, 16, 64), vp=_t(5, 2, 16, 64), lists=_i(3, 2, 4), lens=_i(3, 2), kn=None, vn=None)
    a.update(change)
    with pytest.raises(error):
        bd.bd_attn_paged_sparse_decode_fwd(*a.values())


@pytest.mark.parametrize("change,error", [
    (dict(kp=_t(5, 16, 64)), ValueError), (dict(kp=_t(5, 2, 16, 64, dtype=torch.float32)), TypeError), (dict(table=_i(2, 4)), ValueError),
    (dict(kp=_t(5, 2, 16, 128)[..., ::2]), ValueError), (dict(before=_i(2)), ValueError), (dict(before=_t(3)), TypeError),
    (dict(s=_t(5, 2, 1, 64)), ValueError), (dict(s=_t(5, 2, 2, 64, dtype=torch.float32)), TypeError),
    (dict(s=_t(2, 5, 2, 64).transpose(0, 1)), ValueError),
])
def test_summarize_binding_refusals(change, error):
    a = dict(kp=_t(5, 2, 16, 64), table=_i(3, 4), before=_i(3), lens=_i(3), s=_t(5, 2, 2, 64))
    a.update(change)
    with pytest.raises(error):
        bd.bd_paged_summarize(*a.values())


@pytest.mark.parametrize("change,error", [
    (dict(q=_t(3, 4, 64)), ValueError), (dict(q=_t(3, 4, 1, 64, dtype=torch.float16)), TypeError), (dict(s=_t(5, 2, 64)), ValueError),
    (dict(s=_t(5, 2, 2, 128)), ValueError), (dict(s=_t(5, 2, 3, 64)), ValueError), (dict(table=_i(2, 4)), ValueError), (dict(lens=_i(4)), ValueError),
    (dict(budget=0), ValueError), (dict(budget=1.5), TypeError), (dict(P=1 << 32), ValueError), (dict(budget=(1 << 32) + 2), ValueError),
])
def test_select_binding_refusals(change, error):
    a = dict(q=_t(3, 4, 1, 64), s=_t(5, 2, 2, 64), table=_i(3, 4), lens=_i(3), P=16, budget=2)
    a.update(change)
    with pytest.raises(error):
        bd.bd_paged_select(*a.values())
