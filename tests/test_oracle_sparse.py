"""Pins of the oracle of decoding with shared prefixes, of page summaries, of the
choice of pages and of decoding over lists (CPU): against the paged oracle and
against what the definitions imply."""
import itertools

import numpy as np

import oracle


def _cache(rng, n, H, P, D):
    return rng.normal(size=(2, n, H, P, D))


def test_shared_decode_is_paged_decode_of_the_joined_tables():
    """Prefixes of whole pages: each sequence's table is the prefix's pages, then its own."""
    rng = np.random.default_rng(1)
    Hq, Hkv, S, D, P = 4, 2, 3, 64, 16
    kp, vp = _cache(rng, 20, Hkv, P, D)
    sizes, prefix_lens, prefix = [2, 0, 1], [32, 16, 48], rng.permutation(20)[:9].reshape(3, 3)
    table, lens = rng.permutation(20)[:8].reshape(4, 2), [5, 0, 32, 17]
    q, (kn, vn) = rng.normal(size=(4, Hq, S, D)), rng.normal(size=(2, 4, Hkv, S, D))
    joined = [list(prefix[0][:2]) + list(table[0]), list(prefix[0][:2]) + list(table[1]), list(prefix[2]) + list(table[2]),
              list(table[3])]
    total = [32 + 5, 32, 48 + 32, 17]
    joined = np.array([r + [-1] * (5 - len(r)) for r in joined])
    for new in ((kn, vn), (None, None)):
        got = oracle.shared_decode_forward(q, kp, vp, sizes, prefix, prefix_lens, table, lens, *new)
        want = oracle.paged_decode_forward(q, kp, vp, joined, total, *new)
        for a, b in zip(got, want):
            np.testing.assert_allclose(a, b, atol=1e-12)


def test_groups_end_with_the_sequences():
    """Sizes past the sequences are cut there, and negative ones are 0."""
    rng = np.random.default_rng(2)
    kp, vp = _cache(rng, 6, 1, 16, 64)
    q = rng.normal(size=(3, 1, 1, 64))
    prefix, table = np.array([[0], [1], [2]]), np.array([[3], [4], [5]])
    a = oracle.shared_decode_forward(q, kp, vp, [-4, 2, 99], prefix, [16, 16, 16], table, [1, 2, 3])
    b = oracle.shared_decode_forward(q, kp, vp, [0, 2, 1], prefix, [16, 16, 16], table, [1, 2, 3])
    assert all((x == y).all() for x, y in zip(a, b))


def test_scores_bound_every_key():
    """A row's bound is at least each of its products, and is reached where a page holds one key."""
    rng = np.random.default_rng(3)
    P, D = 16, 64
    kp = rng.normal(size=(5, 2, P, D))
    s = oracle.summarize(kp, np.arange(5)[None], [0], [5 * P], np.zeros((5, 2, 2, D)))
    q = rng.normal(size=(7, D))
    for h, r in itertools.product(range(2), range(7)):
        assert (oracle.page_scores(q[r:r + 1], s[:, h], range(5)) >= (kp[:, h] @ q[r]).max(axis=1) - 1e-12).all()
    one = oracle.summarize(kp, np.arange(5)[None], [0], [1], np.zeros((5, 2, 2, D)))
    np.testing.assert_allclose(oracle.page_scores(q, one[:, 1], [0])[0], (kp[0, 1, 0] @ q.T).sum(), rtol=1e-12)
    assert (one[1:] == 0).all()


def test_summaries_follow_the_cache():
    """Token by token or at once, the same summaries; pages of no new token stay."""
    rng = np.random.default_rng(4)
    kp, table = rng.normal(size=(6, 1, 16, 8)), np.array([[4, 1, 5]])
    at_once = oracle.summarize(kp, table, [0], [40], np.zeros((6, 1, 2, 8)))
    steps = np.zeros((6, 1, 2, 8))
    for n in range(40):
        steps = oracle.summarize(kp, table, [n], [n + 1], steps)
    assert (steps == at_once).all() and (at_once[[0, 2, 3]] == 0).all()
    np.testing.assert_array_equal(at_once[5, 0, 1], kp[5, 0, :8].max(axis=0))


def test_no_new_position_no_summary():
    """[from, len) names no position: nothing is written, inside a page as at its edge, and where from is past len."""
    rng = np.random.default_rng(8)
    kp, table = rng.normal(size=(4, 1, 16, 8)), np.array([[2, 0, 3]])
    mark = np.full((4, 1, 2, 8), 7.0)
    for before, after in ((20, 20), (16, 16), (32, 20), (21, 20), (48, 48), (99, 50), (0, 0), (3, -1), (1 << 30, 1 << 30)):
        assert (oracle.summarize(kp, table, [before], [after], mark) == mark).all(), (before, after)
    one = oracle.summarize(kp, table, [20], [21], mark)
    np.testing.assert_array_equal(one[0, 0], [kp[0, 0, :5].min(axis=0), kp[0, 0, :5].max(axis=0)])
    assert (one[1:] == mark[1:]).all()


def test_choice_of_pages():
    """By hand: the first and the last page, then the highest scores, the earlier of equal ones; keys of the last page."""
    D = 64
    s = np.zeros((8, 1, 2, D))
    for page, x in enumerate([0, 5, 9, 5, 9, 1, 7, 2]):
        s[page, 0, 1, 0] = x
    q = np.ones((1, 1, 1, D))
    table = np.array([[7, 6, 5, 4, 3, 2, 1, 0]])  # scores 2 7 1 9 5 9 5 0
    for budget, first, last, want, keys in [
        (4, 1, 1, [7, 4, 2, 0], 3 * 16 + 3), (3, 0, 0, [6, 4, 2], 48), (5, 0, 0, [6, 4, 3, 2, 1], 80), (4, 0, 0, [6, 4, 3, 2], 64),
        (1, 0, 1, [0], 3), (2, 0, 2, [1, 0], 19), (9, 0, 0, [7, 6, 5, 4, 3, 2, 1, 0, -1], 7 * 16 + 3),
    ]:
        lists, n = oracle.select(q, s, table, [7 * 16 + 3], 16, budget, first, last)
        assert lists[0, 0].tolist() == want and n[0, 0] == keys
    lists, n = oracle.select(q, s, np.array([[7, -1, 5, 99]]), [64], 16, 3, 1, 1)
    assert lists[0, 0].tolist() == [7, 5, -1] and n[0, 0] == 32


def test_lists_of_all_pages_are_paged_decode():
    rng = np.random.default_rng(5)
    kp, vp = _cache(rng, 9, 2, 16, 64)
    table, lens = np.array([[0, 3, 5], [8, 1, 2]]), [37, 16]
    q, (kn, vn) = rng.normal(size=(2, 4, 2, 64)), rng.normal(size=(2, 2, 2, 2, 64))
    want = oracle.paged_decode_forward(q, kp, vp, table, lens, kn, vn)
    got = oracle.sparse_decode_forward(q, kp, vp, table[:, None].repeat(2, 1), np.array(lens)[:, None].repeat(2, 1), kn, vn)
    for a, b in zip(got, want):
        np.testing.assert_allclose(a, b, atol=1e-12)
