"""GPU parity of the head norms with rotation against the fp64 oracle.

Tolerances.  Results are computed in float32 and rounded once: in bfloat16 by at
most half a step, 2^-8 of the value.  The float32 part is some twenty roundings
of 2^-24 relative to the row's largest value (the row's sum of squares and the
mean of h n, over 128 values in a tree, weigh less): below 1e-5 of it.  A
weight's gradient is a float32 sum of at most 400 dependent additions (8 heads,
3 + 4 over a workgroup, one per 32 of at most 10^4 workgroups, 32): below 400 *
2^-24 = 2.4e-5 of the sum of the absolute terms.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_22234_amd as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, tag, half_step=True):
    want = np.broadcast_to(want, got.shape)
    tol = 1e-5 * np.abs(want).max(-1, keepdims=True) + (2.0 ** -8 * np.abs(want) if got.dtype == BF else 0.0)
    err = np.abs(_np(got) - want)
    print(f"[rope] {tag}: largest error / tolerance {float((err / (tol + 1e-30)).max()):.3f}", flush=True)
    assert (err <= tol).all()


def _sum_close(got, want, terms, tag):
    tol = 2.4e-5 * terms + (2.0 ** -8 * np.abs(want) if got.dtype == BF else 0.0)
    err = np.abs(_np(got) - want)
    print(f"[rope] {tag}: largest error / tolerance {float((err / (tol + 1e-30)).max()):.3f}", flush=True)
    assert (err <= tol).all()


def _case(B, N, Hq, Hkv, D, dt, wdt, seed, n_rope=500):
    g = torch.Generator().manual_seed(seed)

    def rows(*shape):
        return torch.randn(shape, generator=g).to(dt)

    c = dict(qkv=rows(B, N, (Hq + 2 * Hkv) * D), wq=(1 + 0.3 * torch.randn(D, generator=g)).to(wdt),
             wk=(1 + 0.3 * torch.randn(D, generator=g)).to(wdt),
             pos=torch.randint(0, n_rope, (B, N), generator=g, dtype=torch.int32),
             dq=rows(B, Hq, N, D), dk=rows(B, Hkv, N, D), dv=rows(B, Hkv, N, D))
    c = {k: v.to(DEV) for k, v in c.items()}
    c["rope"] = bd.bd_rope_table(n_rope, D, device=DEV)
    return c


def _qkv_views(qkv, Hq, Hkv, D):
    return qkv.unflatten(-1, (Hq + 2 * Hkv, D)).split([Hq, Hkv, Hkv], dim=-2)


def _parts(c, Hq, Hkv, D):
    return _qkv_views(c["qkv"], Hq, Hkv, D)


CASES = [
    # B, N, Hq, Hkv, D, rows, weights
    (1, 1, 1, 1, 64, BF, BF),            # one token, one head
    (1, 1, 5, 2, 128, F32, F32),
    (3, 33, 4, 2, 128, BF, F32),         # a workgroup's tokens across sequences, ragged end
    (2, 64, 3, 1, 64, BF, BF),           # heads that no run divides, Hq not a multiple of Hkv * 2
    (1, 1000, 32, 8, 128, BF, BF),       # several heads a workgroup
    (5, 131, 16, 16, 64, F32, F32),
    (2, 2500, 32, 8, 64, BF, F32),
    (1, 4100, 7, 3, 128, BF, F32),       # runs of two heads, a last one of one
    (3, 3000, 11, 5, 64, F32, F32),      # ... of four, a last one of three and of one
]


@pytest.mark.parametrize("B,N,Hq,Hkv,D,dt,wdt", CASES)
def test_matches_oracle(B, N, Hq, Hkv, D, dt, wdt):
    print(f"[rope] B{B} N{N} H{Hq}/{Hkv} D{D} {dt} {wdt}", flush=True)
    c = _case(B, N, Hq, Hkv, D, dt, wdt, seed=B * N + D)
    q, k, v = _parts(c, Hq, Hkv, D)
    rest = (c["wq"], c["wk"], c["rope"], c["pos"])
    qo, ko, vo = bd.bd_qk_norm_rope_fwd(q, k, v, *rest)
    table, pos = _np(c["rope"]), c["pos"].cpu().numpy()
    _close(qo, oracle.norm_rope(_np(q), _np(c["wq"]), table, pos, 1e-6), "q")
    _close(ko, oracle.norm_rope(_np(k), _np(c["wk"]), table, pos, 1e-6), "k")
    assert torch.equal(vo, v.transpose(1, 2)) and all(t.is_contiguous() for t in (qo, ko, vo))
    gq, gk, gv, gwq, gwk = bd.bd_qk_norm_rope_bwd(c["dq"], c["dk"], c["dv"], q, k, *rest)
    for got, gw, d, x, w, tag in ((gq, gwq, c["dq"], q, c["wq"], "q"), (gk, gwk, c["dk"], k, c["wk"], "k")):
        dx, dw, terms = oracle.norm_rope_backward(_np(d), _np(x), _np(w), table, pos, 1e-6)
        _close(got, dx, "d" + tag)
        _sum_close(gw, dw, terms, "dw" + tag)
    assert torch.equal(gv, c["dv"].transpose(1, 2))


def test_table_matches_float64_angles():
    """Rows far out, also with frequencies given: cos and sin of float64 angles, rounded once."""
    D, n = 128, 300000
    t = bd.bd_rope_table(n, D, theta=1e4, device=DEV)
    rows = np.r_[0:5, 1000:1005, n - 5:n]
    want = oracle.rope_table(n, D, 1e4)[rows]
    # half a step of the value, and the device's sincos: within 1e-9 of the float64 one for such angles
    assert (np.abs(_np(t)[rows] - want) <= 2.0 ** -24 * np.abs(want) + 1e-9).all()
    f = torch.rand(32, dtype=torch.float64, device=DEV)
    t = bd.bd_rope_table(77, 64, inv_freq=f)
    want = oracle.rope_table(77, 64, inv_freq=_np(f))
    assert (np.abs(_np(t) - want) <= 2.0 ** -24 * np.abs(want) + 1e-9).all()


def test_layouts_give_the_same():
    """Separate projections, a fused one, head-major sources, values shared by
    all sequences (stride 0), shared positions, and packed tokens: bitwise."""
    B, N, Hq, Hkv, D = 2, 70, 4, 2, 128
    c = _case(B, N, Hq, Hkv, D, BF, BF, seed=9)
    c["pos"] = c["pos"][:1].expand(B, N).contiguous()
    q, k, v = _parts(c, Hq, Hkv, D)
    v = v[:1].expand(B, N, Hkv, D)
    rest = (c["wq"], c["wk"], c["rope"])
    want = bd.bd_qk_norm_rope_fwd(q, k, v.contiguous(), *rest, c["pos"])
    sources = [
        (q.contiguous(), k.contiguous(), v),
        tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v)),   # [B, H, N, D] in memory
        (q, k.transpose(0, 1).contiguous().transpose(0, 1), v),                      # [N, B, H, D]
    ]
    for s in sources:
        for pos in (c["pos"], c["pos"][0].contiguous()):
            got = bd.bd_qk_norm_rope_fwd(*s, *rest, pos)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    for b in range(B):
        got = bd.bd_qk_norm_rope_fwd(q[b], k[b], v[b], *rest, c["pos"][b])
        assert all(torch.equal(a, w[b]) for a, w in zip(got, want))
    # gradients into views of one fused array
    d = (c["dq"], c["dk"], c["dv"])
    want = bd.bd_qk_norm_rope_bwd(*d, q, k, *rest, c["pos"])
    fused = torch.full((B, N, (Hq + 2 * Hkv) * D + 64), 7.0, dtype=BF, device=DEV)
    views = _qkv_views(fused[..., :-64], Hq, Hkv, D)
    got = bd.bd_qk_norm_rope_bwd(*d, q, k, *rest, c["pos"], 1e-6, *views)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (fused[..., -64:] == 7.0).all()      # nothing past a token's heads


@pytest.mark.parametrize("order", ["head by head", "keys and values", "by sequence", "tokens inside", "heads inside"])
def test_gradients_into_interleaved_arrays(order):
    """The three gradients as views of one array that holds them head by head, sequence by
    sequence, or with tokens or heads innermost: bitwise those of separate arrays."""
    B, N, H, D = 2, 70, 3, 64
    c = _case(B, N, H, H, D, BF, F32, seed=21)
    q, k, v = _parts(c, H, H, D)
    args = (c["dq"], c["dk"], c["dv"], q, k, c["wq"], c["wk"], c["rope"], c["pos"], 1e-6)

    def fused(*shape):
        return torch.full(shape, 7.0, dtype=BF, device=DEV)

    if order == "head by head":
        views = fused(B, N, H, 3, D).unbind(3)
    elif order == "keys and values":
        views = (fused(B, N, H, D), *fused(B, N, H, 2, D).unbind(3))
    elif order == "by sequence":
        views = fused(B, 3, N, H, D).unbind(1)
    elif order == "tokens inside":
        views = [t.transpose(1, 2) for t in fused(B, H, 3, N, D).unbind(2)]
    else:
        views = [t.transpose(0, 1) for t in fused(N, 3, B, H, D).unbind(1)]
    want = bd.bd_qk_norm_rope_bwd(*args)
    got = bd.bd_qk_norm_rope_bwd(*args, *views)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("N,dt", [(9000, BF), (17500, BF), (6000, F32)])
def test_large_calls(N, dt):
    """Calls of more than 64 and 128 MiB (nontemporal loads, and stores), eight heads a
    workgroup: bitwise the results of the same tokens in calls of 500, sampled
    tokens against the oracle; the weights' gradients against sums in float64."""
    Hq, Hkv, D = 10, 3, 128
    c = _case(1, N, Hq, Hkv, D, dt, F32, seed=16)
    q, k, v = _parts(c, Hq, Hkv, D)
    w, d = (c["wq"], c["wk"], c["rope"]), (c["dq"], c["dk"], c["dv"])
    out = bd.bd_qk_norm_rope_fwd(q, k, v, *w, c["pos"])
    grads = bd.bd_qk_norm_rope_bwd(*d, q, k, *w, c["pos"])
    dw = [torch.zeros(D, dtype=torch.float64, device=DEV) for _ in range(2)]
    for n in range(0, N, 500):
        part = slice(n, n + 500)
        pos = c["pos"][:, part].contiguous()
        got = bd.bd_qk_norm_rope_fwd(q[:, part], k[:, part], v[:, part], *w, pos)
        assert all(torch.equal(a, b[:, :, part]) for a, b in zip(got, out))
        got = bd.bd_qk_norm_rope_bwd(*(t[:, :, part].contiguous() for t in d), q[:, part], k[:, part], *w, pos)
        assert all(torch.equal(a, b[:, part]) for a, b in zip(got[:3], grads[:3]))
        dw = [a + b.double() for a, b in zip(dw, got[3:])]
    pick = torch.tensor([0, 31, 32, N // 2, N - 1], device=DEV)
    table, pos = _np(c["rope"]), c["pos"][:, pick].cpu().numpy()
    _close(out[0][:, :, pick], oracle.norm_rope(_np(q[:, pick]), _np(c["wq"]), table, pos, 1e-6), "large q")
    dx, _, _ = oracle.norm_rope_backward(_np(c["dk"][:, :, pick]), _np(k[:, pick]), _np(c["wk"]), table, pos, 1e-6)
    _close(grads[1][:, pick], dx, "large dk")
    # both sides within 2.4e-5 of the sum of the terms' absolute values, here about N H of order 1 each
    for got, want, H in zip(grads[3:], dw, (Hq, Hkv)):
        assert float((got.double() - want).abs().max()) <= 2 * 2.4e-5 * N * H


def test_positions_are_clamped_and_zero_rows_finite():
    D = 64
    c = _case(1, 6, 2, 1, D, F32, F32, seed=10, n_rope=20)
    c["pos"] = torch.tensor([[-5, 0, 19, 20, 1 << 30, -(1 << 31)]], dtype=torch.int32, device=DEV)
    c["qkv"][0, 2] = 0
    q, k, v = _parts(c, 2, 1, D)
    rest = (c["wq"], c["wk"], c["rope"], c["pos"])
    qo, _, _ = bd.bd_qk_norm_rope_fwd(q, k, v, *rest)
    table, pos = _np(c["rope"]), c["pos"].cpu().numpy().astype(np.int64)
    _close(qo, oracle.norm_rope(_np(q), _np(c["wq"]), table, pos, 1e-6), "clamped")
    assert (qo[0, :, 2] == 0).all()
    gq = bd.bd_qk_norm_rope_bwd(c["dq"], c["dk"], c["dv"], q, k, *rest)[0]
    _close(gq, oracle.norm_rope_backward(_np(c["dq"]), _np(q), _np(c["wq"]), table, pos, 1e-6)[0], "clamped dq")


def test_extreme_values():
    """Rows whose squares leave bfloat16 but not float32, tiny rows under eps."""
    D = 128
    c = _case(1, 4, 1, 1, D, BF, BF, seed=11)
    x = c["qkv"].view(1, 4, 3, D)
    x[0, 0] *= 1e15
    x[0, 1] *= 1e-15
    x[0, 2, :, 1:] = 0
    q, k, v = _parts(c, 1, 1, D)
    rest = (c["wq"], c["wk"], c["rope"], c["pos"])
    qo, ko, _ = bd.bd_qk_norm_rope_fwd(q, k, v, *rest)
    for got, src, w in ((qo, q, "wq"), (ko, k, "wk")):
        _close(got, oracle.norm_rope(_np(src), _np(c[w]), _np(c["rope"]), c["pos"].cpu().numpy(), 1e-6), "extreme")


def test_no_tokens():
    w = torch.ones(64, device=DEV)
    rope = bd.bd_rope_table(4, 64, device=DEV)
    q, k = torch.empty((2, 0, 3, 64), device=DEV), torch.empty((2, 0, 1, 64), device=DEV)
    pos = torch.empty((2, 0), dtype=torch.int32, device=DEV)
    out = bd.bd_qk_norm_rope_fwd(q, k, k, w, w, rope, pos)
    assert [tuple(t.shape) for t in out] == [(2, 3, 0, 64), (2, 1, 0, 64), (2, 1, 0, 64)]
    *_, gwq, gwk = bd.bd_qk_norm_rope_bwd(*out, q, k, w, w, rope, pos)
    assert (gwq == 0).all() and (gwk == 0).all()


@pytest.mark.parametrize("fused", [True, False])
def test_autograd(fused):
    """Gradients through autograd are the backward call's; a result that no loss uses counts as zeros."""
    B, N, Hq, Hkv, D = 2, 40, 4, 2, 64
    c = _case(B, N, Hq, Hkv, D, F32, F32, seed=12)
    q, k, v = _parts(c, Hq, Hkv, D)
    rest = (c["wq"].requires_grad_(), c["wk"].requires_grad_(), c["rope"], c["pos"])
    if fused:
        ins = (c["qkv"].requires_grad_(), *rest[:2])
        out = bd.qkv_norm_rope(c["qkv"], Hq, Hkv, *rest)
    else:
        q, k, v = (t.contiguous().requires_grad_() for t in (q, k, v))
        ins = (q, k, v, *rest[:2])
        out = bd.qk_norm_rope(q, k, v, *rest)
    for dv in (c["dv"], None):
        loss = (out[0] * c["dq"]).sum() + (out[1] * c["dk"]).sum() + (0 if dv is None else (out[2] * dv).sum())
        got = torch.autograd.grad(loss, ins, retain_graph=True)
        zero = torch.zeros_like(c["dv"])
        gq, gk, gv, gwq, gwk = bd.bd_qk_norm_rope_bwd(c["dq"], c["dk"], zero if dv is None else dv, q, k, *rest)
        want = (torch.cat([gq, gk, gv], 2).view(B, N, -1),) if fused else (gq, gk, gv)
        assert all(torch.equal(a, b) for a, b in zip(got, (*want, gwq, gwk)))
    with pytest.raises(RuntimeError):
        g = torch.autograd.grad((out[0] * c["dq"]).sum(), ins[0], create_graph=True)[0]
        g.sum().backward()


def test_same_bits_twice_and_on_another_stream():
    c = _case(2, 777, 16, 4, 128, BF, F32, seed=13)
    q, k, v = _parts(c, 16, 4, 128)
    rest = (c["wq"], c["wk"], c["rope"], c["pos"])

    def both(stream=None):
        return (*bd.bd_qk_norm_rope_fwd(q, k, v, *rest, stream=stream),
                *bd.bd_qk_norm_rope_bwd(c["dq"], c["dk"], c["dv"], q, k, *rest, stream=stream))

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [both(), both(side)]
    with torch.cuda.stream(side):
        got.append(both())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_guard_rows_stay():
    """Nothing is written in front of or behind the results."""
    B, N, Hq, Hkv, D = 1, 37, 3, 1, 64
    c = _case(B, N, Hq, Hkv, D, BF, BF, seed=14)
    q, k, v = _parts(c, Hq, Hkv, D)

    def guarded(*shape):
        n = int(np.prod(shape))
        t = torch.full((n + 256,), 5.0, dtype=BF, device=DEV)
        return t, t[128:128 + n].view(shape)

    (a, qo), (b, ko), (d, vo) = guarded(B, Hq, N, D), guarded(B, Hkv, N, D), guarded(B, Hkv, N, D)
    bd.bd_qk_norm_rope_fwd(q, k, v, c["wq"], c["wk"], c["rope"], c["pos"], 1e-6, qo, ko, vo)
    for t in (a, b, d):
        assert (t[:128] == 5).all() and (t[-128:] == 5).all()


def test_graph_replays():
    """Forward and backward captured, replayed with new inputs and eager work between."""
    B, N, Hq, Hkv, D = 1, 300, 8, 2, 128
    c = _case(B, N, Hq, Hkv, D, BF, F32, seed=15)
    q, k, v = _parts(c, Hq, Hkv, D)
    rest = (c["wq"], c["wk"], c["rope"], c["pos"])

    def both():
        return (*bd.bd_qk_norm_rope_fwd(q, k, v, *rest),
                *bd.bd_qk_norm_rope_bwd(c["dq"], c["dk"], c["dv"], q, k, *rest))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for i in range(3):
        c["qkv"].normal_()
        c["dq"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, both()))
