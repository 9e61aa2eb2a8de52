"""Pins of the oracle of the head norms with rotation, of paged decoding and of
the page tables (CPU): against differences, against the dense decode oracle,
and against what a page table has to satisfy."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("D,eps", [(64, 1e-6), (128, 1e-2)])
def test_norm_rope_gradient_matches_differences(D, eps):
    """Central differences of the float64 forward in random directions: error
    h^2 / 6 times the third derivative (|x| of order 1, so of order 1e3 at most)
    plus 2^-52 / h of the values' rounding: 1e-7 at h = 1e-5."""
    rng = np.random.default_rng(3)
    B, N, H = 2, 3, 2
    x, w = rng.normal(size=(B, N, H, D)), 1 + 0.3 * rng.normal(size=D)
    d = rng.normal(size=(B, H, N, D))
    pos = rng.integers(0, 50, (B, N))
    table = oracle.rope_table(50, D)
    dx, dw, _ = oracle.norm_rope_backward(d, x, w, table, pos, eps)
    h = 1e-5
    for _ in range(4):
        ux, uw = rng.normal(size=x.shape), rng.normal(size=D)
        hi, lo = ((d * oracle.norm_rope(x + s * ux, w + s * uw, table, pos, eps)).sum() for s in (h, -h))
        want = (dx * ux).sum() + (dw * uw).sum()
        assert abs((hi - lo) / (2 * h) - want) <= 1e-7 * max(1.0, np.abs(dx * ux).sum() + np.abs(dw * uw).sum())


def test_norm_rope_keeps_what_it_must():
    """Norms of the outputs: sqrt(D) with unit weights (the rotation keeps them);
    position 0 rotates nothing; scores depend on the difference of positions only."""
    rng = np.random.default_rng(4)
    D = 64
    x = rng.normal(size=(5, 1, D))
    t = oracle.rope_table(40, D)
    y = oracle.norm_rope(x, np.ones(D), t, np.array([0, 7, 9, 17, 39]), 0.0)
    np.testing.assert_allclose((y * y).sum(-1), D, rtol=1e-12)
    np.testing.assert_allclose(y[0, 0], x[0, 0] / np.sqrt((x[0, 0] ** 2).mean()), rtol=1e-12)
    q, k = (oracle.norm_rope(np.repeat(a[None, None], 3, 0), np.ones(D), t, np.array(p), 0.0)[0]
            for a, p in ((x[0, 0], [5, 12, 30]), (x[1, 0], [2, 9, 27])))
    np.testing.assert_allclose((q * k).sum(-1), (q[0] * k[0]).sum(), rtol=1e-10)


def test_paged_decode_matches_dense_decode():
    rng = np.random.default_rng(5)
    B, Hq, Hkv, S, D, P, width = 3, 4, 2, 3, 64, 16, 4
    lens = [0, 17, 64]
    kc, vc = rng.normal(size=(2, B, Hkv, width * P, D))
    order = rng.permutation(B * width)
    table = order.reshape(B, width)
    kp, vp = np.empty((2, B * width, Hkv, P, D))
    for pages, dense in ((kp, kc), (vp, vc)):
        pages[table] = dense.reshape(B, Hkv, width, P, D).transpose(0, 2, 1, 3, 4)
    q, kn, vn = rng.normal(size=(B, Hq, S, D)), *rng.normal(size=(2, B, Hkv, S, D))
    for new in ((kn, vn), (None, None)):
        o, lse = oracle.paged_decode_forward(q, kp, vp, table, lens, *new)
        if new[0] is not None:
            want = oracle.decode_forward(q, kc, vc, kn, vn, lens)
            np.testing.assert_allclose(o, want[0], atol=1e-12)
            np.testing.assert_allclose(lse, want[1], atol=1e-12)
        else:
            assert (o[0] == 0).all() and np.isneginf(lse[0]).all() and np.isfinite(lse[1:]).all()
    # a page that is none: the softmax over the other keys
    t2 = table.copy()
    t2[2, 1] = -1
    o, _ = oracle.paged_decode_forward(q, kp, vp, t2, lens)
    z = q[2, 0] @ np.delete(kc[2, 0], np.s_[16:32], 0).T / 8.0
    e = np.exp(z - z.max(1, keepdims=True))
    np.testing.assert_allclose(o[2, 0], e @ np.delete(vc[2, 0], np.s_[16:32], 0) / e.sum(1, keepdims=True), atol=1e-12)


@pytest.mark.parametrize("S", [0, 4])
def test_paged_plan_places_every_token_once(S):
    """Three steps in a row: every token has a row of its own, in its sequence's
    pages at its position, and no page serves two sequences."""
    rng = np.random.default_rng(6)
    B, P, width, pages = 5, 16, 8, 40
    table, lens = np.full((B, width), -1), np.zeros(B, dtype=np.int64)
    free, head, owner = rng.permutation(pages), 0, {}
    for _ in range(3):
        new = rng.integers(0, 5 if S else 30, B)
        table, lens2, cu, slots, pos, (head, lost) = oracle.paged_plan(lens, new, table, free, head, pages, P, S, int(new.sum()))
        assert lost == 0
        for b in range(B):
            for i in range(new[b]):
                t = b * S + i if S else cu[b] + i
                assert pos[t] == lens[b] + i and slots[t] == table[b, pos[t] // P] * P + pos[t] % P
                assert slots[t] not in owner
                owner[int(slots[t])] = b
        lens = lens2
    assert all(len({owner[s] for s in owner if s // P == p}) <= 1 for p in range(pages))
    used = sorted(int(p) for p in table[table >= 0])
    assert used == sorted(int(p) for p in free[:head])


def test_paged_plan_past_total_by_hand():
    """12 of 10 + 64 packed tokens have a row: two of the second sequence; its four pages are taken and entered."""
    table, lens, cu, slots, pos, state = oracle.paged_plan([0, 0], [10, 64], [[7, 7, 7, 7], [7, 7, 7, 7]], [3, 0, 9, 5, 1], 0, 6, 16,
                                                           0, 12)
    assert table.tolist() == [[3, 7, 7, 7], [0, -1, 5, 1]]          # (9 is no page)
    assert lens.tolist() == [10, 64] and cu.tolist() == [0, 10, 74] and state.tolist() == [5, 62]
    assert slots.tolist() == [*range(48, 58), 0, 1] and pos.tolist() == [*range(10), 0, 1]
