"""GPU parity of decoding with shared prefixes, of page summaries, of the choice of
pages and of decoding over chosen pages, each against the fp64 oracle, and the
rollouts they make together.

Tolerances (inputs of standard deviation 0.5, D <= 128).  O is rounded to bfloat16,
at most 2^-8 of each value.  Below that, relative to the sum of |p v|: scores are
float32 sums of up to 128 exact products, each sum off by at most 128 * 2^-24 of
sum |q_d k_d| <= 40, scaled by 1 / sqrt(D): 2^-15; P has 16 bits, 2^-17; sums over up to 4096 keys
in steps of 16, 2^-16: 2^-14 in all, which also bounds the LSE's own error.
Summaries and lists have to be equal.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_22234_amd as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16
I32 = dict(dtype=torch.int32, device=DEV)
SUMS = 2.0 ** -14


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _ints(*lists):
    out = [torch.tensor(x, **I32) for x in lists]
    return out[0] if len(out) == 1 else out


def _check(got, want, size, tag):
    (O, L), (Or, Lr) = map(_np, got), want
    seen = np.isfinite(Lr)
    assert (np.isneginf(L) == ~seen).all() and (O[~seen] == 0).all()
    err, tol = np.abs(O - Or), 2.0 ** -8 * np.abs(Or) + SUMS * size
    lse = np.abs(L[seen] - Lr[seen]).max(initial=0.0)
    print(f"[sparse] {tag}: O {float((err / (tol + 1e-30)).max()):.3f} of its tolerance, LSE {lse / SUMS:.3f}", flush=True)
    assert (err <= tol).all() and lse <= SUMS


def _cache(n, Hkv, P, D, order, g):
    def rows(*shape):
        return (torch.randn(shape, generator=g) * 0.5).to(BF).to(DEV)

    if order == "heads":
        return rows(n, Hkv, P, D), rows(n, Hkv, P, D)
    if order == "tokens":
        return tuple(rows(n, P, Hkv, D).permute(0, 2, 1, 3) for _ in range(2))
    kv = rows(n, P, Hkv, 2, D).permute(3, 0, 2, 1, 4)  # K and V of a head side by side
    return kv[0], kv[1]


def _table(lens, P, width, ids):
    """Tables that take the page ids in order, -1 past each length."""
    t = torch.full((len(lens), width), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        k = -(-min(max(n, 0), width * P) // P)
        t[b, :k] = torch.tensor(ids[:k], dtype=torch.int32)
        del ids[:k]
    return t.to(DEV)


def _shared_inputs(sizes, prefix, lens, Hq, Hkv, D, S, P, order, block, seed):
    g = torch.Generator().manual_seed(seed)
    widths = [max(1, max(-(-max(n, 0) // P) for n in x)) + 1 for x in (prefix, lens)]
    n = sum(-(-max(x, 0) // P) for x in prefix + lens) + 3
    kp, vp = _cache(n, Hkv, P, D, order, g)
    ids = torch.randperm(n, generator=g).tolist()
    tables = [_table(x, P, w, ids) for x, w in zip((prefix, lens), widths)]
    B = len(lens)
    q = (torch.randn((B, Hq, S, D), generator=g) * 0.5).to(BF).to(DEV)
    new = [(torch.randn((B, Hkv, S, D), generator=g) * 0.5).to(BF).to(DEV) if block else None for _ in range(2)]
    return [q, kp, vp, _ints(sizes), tables[0], _ints(prefix), tables[1], _ints(lens), *new]


def _shared_oracle(a, absolute=False, scale=None):
    q, kp, vp, sizes, pt, pl, t, ln, kn, vn = a
    v, w = (np.abs(_np(x)) if absolute and x is not None else _np(x) for x in (vp, vn))
    return oracle.shared_decode_forward(_np(q), _np(kp), v, sizes.tolist(), pt.tolist(), pl.tolist(), t.tolist(), ln.tolist(),
                                        _np(kn), w, scale)


def _check_shared(a, got, tag, scale=None):
    _check(got, _shared_oracle(a, scale=scale), _shared_oracle(a, True, scale)[0], tag)


# Group sizes (empty ones, sequences behind the last group, sizes that pass the sequences), prefixes and own keys of no
# key, one key, and around pages and tiles; rows of a group and of a sequence at the edges of waves and teams.
SHARED = [
    # sizes, prefix, own lens, Hq, Hkv, D, S, P, order, block
    ([1], [1], [0], 1, 1, 64, 1, 16, "heads", False),
    ([1], [0], [1], 2, 1, 128, 1, 16, "heads", False),
    ([1], [0], [0], 2, 1, 128, 1, 16, "heads", False),                             # no key at all
    ([8], [300], [1, 0, 16, 17, 31, 32, 33, 64], 8, 2, 128, 1, 16, "tokens", False),  # 32 rows a group
    ([3, 0, 2, 1], [65, 9, 0, 128], [5, 70, 0, 0, 33, 2], 8, 2, 64, 1, 32, "heads", False),
    ([2, -7, 99], [48, 16, 100], [5, 70, 0, 20], 4, 4, 64, 1, 16, "sides", False),
    ([0, 0], [48, 16], [5, 0, 20], 4, 2, 128, 1, 16, "heads", False),              # no sequence in a group
    ([2, 1], [129, 1000], [5, 70, 0, 20, 64], 4, 2, 64, 4, 64, "heads", True),     # two sequences behind the groups
    ([3], [700], [100, 3, 0], 12, 3, 128, 4, 16, "tokens", True),                  # 48 rows: two waves
    ([4], [500], [100, 3, 0, 65], 16, 4, 64, 4, 32, "heads", True),                # 64 rows
    ([5], [500], [100, 3, 0, 65, 1], 16, 4, 128, 4, 32, "heads", True),            # 80 rows
    ([8], [260], [0, 1, 2, 3, 60, 64, 65, 70], 16, 4, 128, 4, 16, "heads", True),  # 128 rows
    ([9], [97], [0, 1, 2, 3, 60, 64, 65, 70, 9], 16, 4, 64, 4, 64, "tokens", True),  # 144 rows
    ([3, 5], [400, 31], [0, 1, 100, 3, 60, 64, 65, 2], 8, 2, 128, 32, 32, "heads", True),   # 384 and 640 rows
    ([4, 1, 2], [90, 1030, 64], [10, 40, 0, 33, 1, 2, 3], 4, 1, 64, 40, 16, "heads", False),  # 160 rows a sequence
    ([1] * 70, [i % 50 for i in range(70)], [i % 37 for i in range(70)], 4, 2, 64, 1, 16, "tokens", True),
    ([30] * 10, [40 * i for i in range(10)], [i % 23 for i in range(300)], 2, 1, 128, 1, 16, "heads", False),
    ([2, 1], [3000, 4096], [17, 900, 64], 8, 8, 128, 1, 256, "tokens", False),
    ([5, 2, 1], [33, 4, 70], [1] * 8, 33, 1, 64, 1, 16, "heads", False),           # 33 rows a sequence
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared_decode_matches_oracle(case):
    print(f"[sparse] shared {SHARED[case]}", flush=True)
    a = _shared_inputs(*SHARED[case], seed=100 + case)
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*a), f"shared {case}")


def test_shared_many_groups():
    """More groups than a workgroup has threads, most of them empty, and wild sizes between."""
    g = np.random.default_rng(6)
    sizes = [int(n) for n in np.where(g.random(700) < 0.5, 0, g.integers(-3, 4, 700))]
    B = 300
    prefix = [int(n) for n in g.integers(0, 80, 700)]
    a = _shared_inputs(sizes, prefix, [int(n) for n in g.integers(0, 40, B)], 4, 2, 64, 1, 16, "heads", False, 7)
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*a), "many groups")


@pytest.mark.parametrize("B", [7, 9])
@pytest.mark.parametrize("wide", [False, True])
def test_shared_lists_that_end_in_empty_groups(B, wide):
    """Members all gone before the list ends, or sequences behind it; an overlong group and empty ones between."""
    sizes = [0, 3, 0, 0, 4] + [0] * 40 + ([5] if B == 7 else [])
    a = _shared_inputs(sizes, [10, 300, 7, 0, 170] + [33] * (len(sizes) - 5), list(range(5, 5 + B)), 32, 2, 128, 32, 16, "heads", True, 17)
    if wide:
        a = _widened(a)
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*a), f"empty end B{B} wide {wide}")


@pytest.mark.parametrize("S,Hq,D,P", [(1, 8, 128, 16), (4, 16, 64, 64), (32, 8, 128, 32)])
def test_shared_absent_pages_clamped_lengths_and_scale(S, Hq, D, P):
    a = _shared_inputs([2, 2], [200, 190], [50, 0, 130, 64], Hq, 2, D, S, P, "heads", S > 1, 11)
    a[4][0, 1] = -1
    a[4][1, : -(-190 // P)] = 1 << 30      # a prefix that is in no page
    a[6][2, 0] = a[1].shape[0]
    a[5] = _ints([200, 1 << 30])
    a[7] = _ints([50, -9, 130, 64])
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*a, scale=0.3), f"absent S{S}", 0.3)


@pytest.mark.parametrize("S,P,order", [(1, 16, "tokens"), (4, 64, "heads"), (32, 32, "sides")])
def test_shared_reads_nothing_else(S, P, order):
    """NaN in every row that no length reaches and wild ids behind the tables' ends: the same bits."""
    a = _shared_inputs([3, 2], [70, 131], [20, 1, 0, 65, 33], 8, 2, 128, S, P, order, S > 1, 13)
    want = bd.bd_attn_paged_shared_decode_fwd(*a)
    keep = torch.zeros(a[1].shape[0], P, dtype=torch.bool)
    for t, lens in ((a[4], a[5].tolist()), (a[6], a[7].tolist())):
        ids = t.cpu()
        for b, n in enumerate(lens):
            for j in range(n):
                keep[ids[b, j // P], j % P] = True
            ids[b, -(-n // P):] = (1 << 31) - 1
        t.copy_(ids)
    for x in a[1:3]:
        x.copy_(torch.where(keep.to(DEV)[:, None, :, None], x, float("nan")))
    got = bd.bd_attn_paged_shared_decode_fwd(*a)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_shared_workspace_streams_and_strided_tables():
    """A workspace full of NaN, tables inside wider arrays, another stream, results in the caller's arrays with
    guards behind them: the same bits."""
    a = _shared_inputs([3, 1, 0, 4], [300, 44, 5, 129], [20, 1, 0, 65, 33, 7, 7, 7], 16, 4, 128, 4, 16, "heads", True, 17)
    want = bd.bd_attn_paged_shared_decode_fwd(*a)
    B, Hq, S, D = a[0].shape
    n = bd.bd_attn_paged_shared_decode_workspace_bytes(B, 4, S, Hq, 4, D, 16, a[4].shape[1], a[6].shape[1])
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    o = torch.full((a[0].numel() + 64,), 7.0, dtype=BF, device=DEV)
    lse = torch.full((B * Hq * S + 64,), 7.0, device=DEV)
    wide = [torch.full((t.shape[0], t.shape[1] + 9), 1 << 20, **I32) for t in (a[4], a[6])]
    for w, t in zip(wide, (a[4], a[6])):
        w[:, 3:3 + t.shape[1]] = t
    b = list(a)
    b[4], b[6] = (w[:, 3:3 + t.shape[1]] for w, t in zip(wide, (a[4], a[6])))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.bd_attn_paged_shared_decode_fwd(*b, out=o[:a[0].numel()].view(a[0].shape), lse=lse[:-64].view(B, Hq, S),
                                             workspace=ws, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (o[-64:] == 7).all() and (lse[-64:] == 7).all()


def test_shared_offsets_past_32_bits():
    """Prefix and own pages behind 2^32 bytes and 2^31 elements of an 8 GiB array."""
    Hq, Hkv, D, P, n = 8, 8, 128, 64, 66000
    kp = torch.empty((n, Hkv, P, D), dtype=BF, device=DEV)
    assert kp.numel() > 1 << 32
    vp = torch.empty_like(kp)
    ids = [n - 1, 5, 32768, 40000, n - 2, 7]
    for x in (kp, vp):
        x[ids] = (torch.randn((6, Hkv, P, D), device=DEV) * 0.5).to(BF)
    q = (torch.randn((2, Hq, 1, D), device=DEV) * 0.5).to(BF)
    rest = [_ints([2]), _ints([ids[:3]]), _ints([150]), _ints([[ids[3]], [ids[4]]]), _ints([64, 30]), None, None]
    small = [x[ids] for x in (kp, vp)]
    near = [_ints([2]), _ints([[0, 1, 2]]), _ints([150]), _ints([[3], [4]]), _ints([64, 30]), None, None]
    got = bd.bd_attn_paged_shared_decode_fwd(q, kp, vp, *rest)
    _check_shared([q, *small, *near], got, "far pages")
    # summaries of far pages, and the choice and decoding of them
    s = torch.zeros((n, Hkv, 2, D), dtype=BF, device=DEV)
    bd.bd_paged_summarize(kp, _ints([ids[:3], ids[3:]]), _ints([0, 0]), _ints([192, 100]), s)
    want = oracle.summarize(_np(small[0]), [[0, 1, 2], [3, 4, 5]], [0, 0], [192, 100], np.zeros((6, Hkv, 2, D)))
    assert (_np(s[ids]) == want).all()
    lists, lens = bd.bd_paged_select(q, s, _ints([ids[:3], ids[3:]]), _ints([192, 100]), P, 2, 0, 1)
    wl, wn = oracle.select(_np(q), want, [[0, 1, 2], [3, 4, 5]], [192, 100], P, 2, 0, 1)
    assert (lists.cpu().numpy() == np.array(ids + [-1])[wl]).all() and (lens.cpu().numpy() == wn).all()
    got = bd.bd_attn_paged_sparse_decode_fwd(q, kp, vp, lists, lens)
    _check_sparse([q, *small, torch.tensor(wl, **I32), lens, None, None], got, "far lists")


def _replayed(call, state, changes):
    """Captures `call` once and replays it after each change of the state in place; every replay against an eager call."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for change in changes:
        change()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), state


def test_shared_decode_replayed():
    """Lengths, group sizes and queries that change between replays."""
    a = _shared_inputs([3, 3, 2], [300, 44, 129], [20, 1, 40, 65, 33, 7, 70, 30], 16, 4, 128, 4, 16, "heads", True, 19)
    _replayed(lambda: bd.bd_attn_paged_shared_decode_fwd(*a), "shared", [
        lambda: None, lambda: a[3].copy_(_ints([1, 5, 2])), lambda: a[5].copy_(_ints([10, 44, 100])),
        lambda: a[7].copy_(_ints([2, 0, 40, 3, 33, 7, 64, 0])), lambda: a[0].mul_(-0.5), lambda: a[3].copy_(_ints([0, 0, 0]))])


# Tables that are much wider than the prefixes in them: with more than 64 rows a group such a call takes its
# prefixes and the sequences' own keys in launches of their own.

def _widened(a):
    b = list(a)
    P, groups = a[1].shape[2], a[4].shape[0]
    b[4] = torch.full((groups, (1 << 20) // P), (1 << 31) - 1, **I32)
    b[4][:, :a[4].shape[1]] = a[4]
    return b


WIDE = [i for i, c in enumerate(SHARED) if len(c[2]) * c[3] // c[4] * c[6] > 64 * len(c[0])] + [-1, -2]
SHARED_MORE = [  # at -1, -2
    ([4, 1], [64 * 37 + 5, 3000], [500, 0, 33, 64, 1], 16, 2, 64, 16, 16, "sides", True),   # 512 and 128 rows
    ([7, 9], [1500, 2049], list(range(0, 160, 10)), 16, 2, 128, 8, 64, "tokens", False),    # 448 and 576 rows
]


@pytest.mark.parametrize("case", WIDE)
def test_shared_wide_tables_match_oracle(case):
    c = SHARED[case] if case >= 0 else SHARED_MORE[-1 - case]
    print(f"[sparse] wide {c}", flush=True)
    a = _shared_inputs(*c, seed=130 + case)
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*_widened(a)), f"wide {case}")


@pytest.mark.parametrize("P,D", [(16, 128), (32, 64), (64, 128)])
def test_shared_wide_tables_absent_pages_and_clamped_lengths(P, D):
    a = _shared_inputs([2, 2], [200, 190], [50, 0, 130, 64], 8, 2, D, 32, P, "heads", True, 11)
    a[4][0, 1] = -1
    a[4][1, : -(-190 // P)] = 1 << 30      # a prefix that is in no page
    a[6][2, 0] = a[1].shape[0]
    a[7] = _ints([50, -9, 130, 64])
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*_widened(a), scale=0.3), f"wide absent P{P}", 0.3)
    a[5] = _ints([-1, 1 << 30])            # to the end of the table, which names no page there
    got = bd.bd_attn_paged_shared_decode_fwd(*_widened(a))
    a[5] = _ints([0, 0])
    _check_shared(a, got, f"wide clamped P{P}")


@pytest.mark.parametrize("P,order", [(16, "tokens"), (64, "heads"), (32, "sides")])
def test_shared_wide_tables_read_nothing_else(P, order):
    a = _shared_inputs([3, 2], [70, 131], [20, 1, 0, 65, 33], 8, 2, 128, 32, P, order, True, 13)
    want = bd.bd_attn_paged_shared_decode_fwd(*_widened(a))
    keep = torch.zeros(a[1].shape[0], P, dtype=torch.bool)
    for t, lens in ((a[4], a[5].tolist()), (a[6], a[7].tolist())):
        for b, n in enumerate(lens):
            for j in range(n):
                keep[int(t[b, j // P]), j % P] = True
    for x in a[1:3]:
        x.copy_(torch.where(keep.to(DEV)[:, None, :, None], x, float("nan")))
    # ... and a workspace full of NaN, another stream, guards behind the results
    w = _widened(a)
    B, Hq, S, D = a[0].shape
    n = bd.bd_attn_paged_shared_decode_workspace_bytes(B, 2, S, Hq, 2, D, P, w[4].shape[1], a[6].shape[1])
    ws = torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV)
    o = torch.full((a[0].numel() + 64,), 7.0, dtype=BF, device=DEV)
    lse = torch.full((B * Hq * S + 64,), 7.0, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.bd_attn_paged_shared_decode_fwd(*w, out=o[:-64].view(a[0].shape), lse=lse[:-64].view(B, Hq, S), workspace=ws[:n],
                                             stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (o[-64:] == 7).all() and (lse[-64:] == 7).all() and (ws[n:] == 255).all()


def test_shared_wide_tables_offsets_past_32_bits():
    Hq, Hkv, D, P, n, S = 32, 8, 128, 64, 66000, 16
    kp = torch.empty((n, Hkv, P, D), dtype=BF, device=DEV)
    vp = torch.empty_like(kp)
    ids = [n - 1, 5, 32768, 40000, n - 2, 7]
    for x in (kp, vp):
        x[ids] = (torch.randn((6, Hkv, P, D), device=DEV) * 0.5).to(BF)
    q = (torch.randn((2, Hq, S, D), device=DEV) * 0.5).to(BF)
    rest = [_ints([2]), _ints([ids[:3]]), _ints([150]), _ints([[ids[3]], [ids[4]]]), _ints([64, 30]), None, None]
    near = [_ints([2]), _ints([[0, 1, 2]]), _ints([150]), _ints([[3], [4]]), _ints([64, 30]), None, None]
    got = bd.bd_attn_paged_shared_decode_fwd(*_widened([q, kp, vp, *rest]))
    _check_shared([q, *(x[ids] for x in (kp, vp)), *near], got, "wide, far pages")


def test_shared_wide_tables_replayed():
    a = _widened(_shared_inputs([3, 3, 2], [300, 44, 129], [20, 1, 40, 65, 33, 7, 70, 30], 16, 4, 128, 16, 16, "heads", True, 19))
    _replayed(lambda: bd.bd_attn_paged_shared_decode_fwd(*a), "shared, wide", [
        lambda: None, lambda: a[3].copy_(_ints([1, 5, 2])), lambda: a[5].copy_(_ints([10, 44, 100])),
        lambda: a[7].copy_(_ints([2, 0, 40, 3, 33, 7, 64, 0])), lambda: a[0].mul_(-0.5), lambda: a[3].copy_(_ints([0, 0, 0]))])


def test_shared_wide_tables_many_groups():
    """More groups than a workgroup has threads, empty ones and wild sizes between, 80 rows a member."""
    g = np.random.default_rng(16)
    sizes = [int(n) for n in g.choice([0, 1, 1, 2, 3, -3], 600)]
    B = sum(max(n, 0) for n in sizes) + 5
    assert B * 80 > 64 * len(sizes)
    prefix = [int(n) for n in g.integers(0, 150, 600)]
    a = _shared_inputs(sizes, prefix, [int(n) for n in g.integers(0, 40, B)], 2, 1, 64, 40, 64, "heads", False, 7)
    _check_shared(a, bd.bd_attn_paged_shared_decode_fwd(*_widened(a)), "wide, many groups")


# Groups that all have the same prefix and queries, with as many key tiles as make the runs' cuts pass 32 bits (2^22), in
# one launch (four rows a group and KV head) and in launches of their own (128 rows).
@pytest.mark.parametrize("groups,n,S,G,P", [(3900, 4, 1, 1, 32), (4000, 4, 1, 1, 32), (8350, 1, 32, 4, 64)])
def test_shared_many_tiles(groups, n, S, G, P):
    Hkv, D, prefix, own = 8, 64, 4000, [1, 64, 33, 40][:n]
    print(f"[sparse] many tiles, {groups} groups of {n}, S{S}", flush=True)
    a = _shared_inputs([n], [prefix], own, Hkv * G, Hkv, D, S, P, "heads", False, 43)
    want, size = _shared_oracle(a), _shared_oracle(a, True)[0]
    for i in (0, 3, 4, 5, 6, 7):
        a[i] = a[i].repeat(groups, *[1] * (a[i].dim() - 1))
    got = bd.bd_attn_paged_shared_decode_fwd(*a)
    _check([x[:n] for x in got], want, size, f"many tiles, {groups} groups")
    # the other groups: off by the same bound, against a result that is off by it
    tol = torch.tensor(2 * (2.0 ** -8 * np.abs(want[0]) + SUMS * size), device=DEV, dtype=torch.float32)
    for o, lse in zip(got[0].split(n * 500), got[1].split(n * 500)):
        assert ((o.view(-1, *tol.shape).float() - got[0][:n].float()).abs() <= tol).all()
        assert ((lse.view(-1, *tol.shape[:3]) - got[1][:n]).abs() <= 2 * SUMS).all()


# ---------------------------------------------------------------------------
# summaries

@pytest.mark.parametrize("B,Hkv,D,P,order,before,after", [
    (1, 1, 64, 16, "heads", [0], [1]), (3, 2, 128, 16, "tokens", [0, 15, 31], [16, 17, 100]),
    (4, 3, 64, 64, "sides", [64, 63, 0, 10], [64, 65, 200, 5]), (2, 8, 128, 256, "heads", [100, 0], [300, 1000]),
    (5, 2, 64, 1024, "tokens", [0, 0, 5, 1023, 2000], [0, 1, 6, 1025, 2049]), (2, 1, 128, 1 << 15, "heads", [0, 40000], [40000, 33000]),
    (300, 4, 128, 32, "heads", [i % 60 for i in range(300)], [i % 90 for i in range(300)]),
    (2, 2, 64, 16, "heads", [-5, 3], [1 << 30, -1]),
    (4200, 5, 64, 16, "tokens", [i % 40 for i in range(4200)], [i % 70 for i in range(4200)]),
])
def test_summaries_match_oracle(B, Hkv, D, P, order, before, after):
    """Equal to the oracle's, and those of other pages as they were; NaN in rows past the lengths."""
    print(f"[sparse] summarize B{B} H{Hkv} D{D} P{P} {order}", flush=True)
    g = torch.Generator().manual_seed(B + P)
    width = 3 if P > 1024 else 8
    real = [min(max(n, 0), width * P) for n in after]
    n = sum(-(-x // P) for x in real) + 3
    kp, _ = _cache(n, Hkv, P, D, order, g)
    table = _table(after, P, width, torch.randperm(n, generator=g).tolist())
    if B > 2:
        table[2, 0] = n if real[2] else -1  # a page that is none
    keys = _np(kp)
    for b, m in enumerate(real):
        if m % P and 0 <= table[b, m // P] < n:
            kp[int(table[b, m // P]), :, m % P:] = float("nan")
    s = torch.full((n, Hkv, 2, D), 3.0, dtype=BF, device=DEV)
    out = bd.bd_paged_summarize(kp, table, *_ints(before, after), s)
    assert out is s
    want = oracle.summarize(keys, table.tolist(), before, after, np.full((n, Hkv, 2, D), 3.0))
    np.testing.assert_array_equal(_np(s), want)


# Sequences without a new position: in the middle of a page, at its edge, truncated ones, lengths past the table.
IDLE = [(20, 20), (16, 16), (32, 20), (21, 20), (128, 128), (1 << 30, 200), (1 << 30, 1 << 30), (0, 0), (5, -1), (9, 3)]


@pytest.mark.parametrize("Hkv,D,P,order", [(1, 64, 16, "heads"), (3, 128, 16, "tokens"), (8, 128, 64, "heads"), (2, 64, 128, "sides")])
def test_summaries_of_idle_sequences_stay(Hkv, D, P, order):
    """Equal lengths before and after: no summary is written; a sequence with one new token between them has its own."""
    print(f"[sparse] idle H{Hkv} D{D} P{P} {order}", flush=True)
    g = torch.Generator().manual_seed(P + D)
    width = 128 // P
    n = (len(IDLE) + 1) * width
    kp, _ = _cache(n, Hkv, P, D, order, g)
    table = torch.arange(n, dtype=torch.int32).view(-1, width).to(DEV)
    before, after = [a for a, _ in IDLE] + [17], [b for _, b in IDLE] + [18]
    s = torch.full((n, Hkv, 2, D), 3.0, dtype=BF, device=DEV)
    bd.bd_paged_summarize(kp, table, *_ints(before, after), s)
    page = len(IDLE) * width + 17 // P
    rows = kp[page, :, : 18 - 17 // P * P]
    assert torch.equal(s[page], torch.stack([rows.amin(1), rows.amax(1)], 1))
    s[page] = 3.0
    assert (s == 3.0).all()


def test_summaries_of_pages_that_an_idle_sequence_gave_away():
    """A finished sequence's last page now belongs to another, which adds to it: the summary is over the owner's keys,
    also in a captured call whose lengths go on."""
    Hkv, D, P, width = 2, 128, 16, 4
    g = torch.Generator().manual_seed(41)
    kp, _ = _cache(40, Hkv, P, D, "heads", g)
    # 64 finished sequences of 20 keys around one that owns their last page, and a fork of it that waits at its first key
    table = torch.tensor([[i % 30, 35, -1, -1] for i in range(64)], **I32)
    table = torch.cat([table[:32], _ints([[34, 35, 36, -1]]), _ints([[33, 35, -1, -1]]), table[32:]])
    lens = [20] * 32 + [31, 17] + [20] * 32
    before, after = _ints(lens, lens)
    before[32] = 30
    s = torch.full((40, Hkv, 2, D), 3.0, dtype=BF, device=DEV)

    def want():
        return torch.tensor(oracle.summarize(_np(kp), table.tolist(), before.tolist(), after.tolist(), np.full(s.shape, 3.0)))

    bd.bd_paged_summarize(kp, table, before, after, s)
    assert (s.double().cpu() == want()).all() and (s[35] != 3.0).all() and (s[:30] == 3.0).all()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.bd_paged_summarize(kp, table, before, after, s)
    for n in (32, 33, 34):
        before[32], after[32] = n - 1, n
        s.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert (s.double().cpu() == want()).all(), n


# ---------------------------------------------------------------------------
# the choice

def _select_check(q, s, table, lens, P, budget, first, last, tag):
    got = bd.bd_paged_select(q, s, table, lens, P, budget, first, last)
    want = oracle.select(_np(q), _np(s), table.tolist(), lens.tolist(), P, budget, first, last)
    print(f"[sparse] select {tag}", flush=True)
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a.cpu().numpy(), b)
    return got


def _select_inputs(B, Hq, Hkv, D, S, P, width, lens, seed):
    g = torch.Generator().manual_seed(seed)
    n = sum(-(-min(max(x, 0), width * P) // P) for x in lens) + 3
    lo, hi = torch.randn((2, n, Hkv, D), generator=g).sort(0)[0]
    s = torch.stack([lo, hi], 2).to(BF).to(DEV)
    q = (torch.randn((B, Hq, S, D), generator=g) * 0.5).to(BF).to(DEV)
    return q, s, _table(lens, P, width, torch.randperm(n, generator=g).tolist()), _ints(lens)


@pytest.mark.parametrize("B,Hq,Hkv,D,S,P,width,lens,budget,first,last", [
    (1, 1, 1, 64, 1, 16, 1, [1], 1, 0, 0), (1, 1, 1, 64, 1, 16, 4, [0], 3, 1, 1),
    (4, 32, 8, 128, 1, 16, 40, [1, 15, 640, 161], 8, 1, 2), (3, 8, 2, 64, 4, 64, 30, [1920, 700, 65], 4, 0, 1),
    (2, 4, 4, 128, 32, 16, 100, [1600, 1599], 16, 2, 0), (2, 12, 3, 64, 3, 32, 300, [9600, 4000], 299, 1, 1),
    (2, 4, 1, 128, 40, 16, 700, [11200, 8209], 33, 0, 33), (1, 8, 8, 64, 1, 16, 2100, [33600], 7, 3, 4),
    (2, 16, 8, 128, 2, 16, 321, [5136, 2049], 40, 1, 2), (33, 2, 1, 64, 1, 16, 321, [i * 155 for i in range(33)], 40, 1, 2),
    # tables far wider than the sequences, and sequences of more pages than LDS holds
    (130, 2, 1, 64, 1, 16, 4100, [65600, 65537, 65536, 0, 1] + [i * 9 for i in range(125)], 40, 1, 2),
    (16, 8, 8, 128, 2, 16, 9000, [140000, 70000, 131073] + [i * 90 for i in range(13)], 50, 1, 2),
    (65, 2, 1, 64, 1, 16, 9000, [140000, 0, 33000] + [i * 50 for i in range(62)], 50, 1, 2),
    (1, 2, 1, 128, 1, 16, 12000, [191999], 2048, 1, 1), (70, 4, 2, 64, 1, 16, 9, [i * 2 for i in range(70)], 5, 1, 1),
    (2, 65, 1, 64, 5, 128, 20, [2560, 100], 20, 0, 0), (3, 4, 2, 64, 1, 16, 10, [-4, 1 << 30, 160], 5, 1, 1),
])
def test_choice_matches_oracle(B, Hq, Hkv, D, S, P, width, lens, budget, first, last):
    a = _select_inputs(B, Hq, Hkv, D, S, P, width, lens, B + width)
    _select_check(*a, P, budget, first, last, f"B{B} H{Hq}/{Hkv} D{D} S{S} P{P} width{width} budget{budget}")


@pytest.mark.parametrize("budget", [1, 5, 64, 100, 513, 600, 1100])
def test_choice_among_equal_scores(budget):
    """Few distinct scores, down to one: the earlier of equal ones; zeros of both signs are equal."""
    P, width = 16, 1200
    q, s, table, lens = _select_inputs(3, 4, 2, 64, 1, P, width, [width * P, width * P - 5, 700 * P], 3)
    kinds = s[:4].clone()
    for i in range(s.shape[0]):
        s[i] = kinds[(i * 7) % 4]
    _select_check(q, s, table, lens, P, budget, 0, 1, f"ties budget{budget}")
    s.copy_(kinds[0].expand_as(s))
    _select_check(q, s, table, lens, P, budget, 1, 0, f"all equal budget{budget}")
    s.zero_()
    s[::3] = -0.0
    _select_check(q, s, table, lens, P, budget, 0, 0, f"zeros budget{budget}")


# Each form of the choice: one workgroup a list with up to 1024, up to 4096 and more pages in the table (the last with lists
# that it holds in LDS and lists that it does not), and several workgroups a list, whose keys the second launch holds in LDS or not.
FORMS = [  # B, Hkv, D, width, lengths in pages
    (3, 2, 64, 40, [40, 39, 17]), (64, 2, 128, 1024, [1024, 1023, 513, 40]), (64, 2, 64, 1025, [1025, 1024, 1000, 513, 41]),
    (16, 8, 128, 2000, [2000, 1999, 1025, 9, 40]), (130, 1, 64, 4096, [4096, 4095, 2049, 40, 8]),
    (32, 4, 128, 4096, [4096, 4095, 0, 41]), (64, 2, 64, 4097, [4097, 4096, 600, 1]), (16, 8, 128, 9000, [9000, 4097, 4096]),
    (3, 2, 64, 700, [700, 699, 513]), (2, 4, 128, 5000, [5000, 4096]), (1, 8, 64, 4097, [4097]),
]


def _form(B, Hkv, D, width, pages, S=1, G=1, seed=5):
    """Inputs of the first lists as given (the odd ones end inside a page), and of short ones behind them."""
    lens = [16 * p - 5 * (i % 2) if p else 0 for i, p in enumerate(pages)] + [(37 * i) % 900 for i in range(B - len(pages))]
    return _select_inputs(B, G * Hkv, Hkv, D, S, 16, width, lens, seed + width)


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_choice_in_each_form(form):
    a = _form(*FORMS[form], S=3, G=2)
    for budget, first, last in ((1, 0, 0), (40, 1, 2), (min(2000, FORMS[form][3]), 2, 5)):
        _select_check(*a, 16, budget, first, last, f"form {FORMS[form]} budget{budget}")


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_choice_among_equal_scores_in_each_form(form):
    q, s, table, lens = _form(*FORMS[form])
    kinds = s[:4].clone()
    for i in range(4):
        s[i::4] = kinds[i * 3 % 4]
    for budget in (1, 37, 600, 1100):
        _select_check(q, s, table, lens, 16, budget, 0, 1 if budget > 1 else 0, f"ties, form {FORMS[form]} budget{budget}")
    s.copy_(kinds[0].expand_as(s))
    _select_check(q, s, table, lens, 16, 515, 1, 0, f"all equal, form {FORMS[form]}")
    s.zero_()
    s[::3] = -0.0
    _select_check(q, s, table, lens, 16, 100, 0, 0, f"zeros, form {FORMS[form]}")


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_choice_with_absent_pages_in_each_form(form):
    """A third of the pages outside the pool, and a list of which fewer than the budget are inside."""
    q, s, table, lens = _form(*FORMS[form])
    g = torch.Generator().manual_seed(form)
    for value in (-1, s.shape[0], -(1 << 31), (1 << 31) - 1):
        table[(torch.rand(table.shape, generator=g) < 0.1).to(DEV)] = value
    table[0, 7 : table.shape[1] - 3] = -1
    for budget, first, last in ((30, 1, 2), (600, 0, 0)):
        _select_check(q, s, table, lens, 16, budget, first, last, f"absent, form {FORMS[form]} budget{budget}")


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_choice_in_each_form_workspace_streams_and_replays(form):
    """A workspace full of ones with guards behind it and behind the results, another stream, and replays of a captured call
    with other lengths, queries and summaries: the same lists."""
    B, Hkv, D, width, _ = FORMS[form]
    a = _form(*FORMS[form])
    budget = 45
    want = bd.bd_paged_select(*a, 16, budget)
    n = bd.bd_paged_select_workspace_bytes(B, 1, Hkv, Hkv, D, 16, width, budget)
    ws = torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV)
    lists, lens = torch.full((B * Hkv * budget + 16,), 7, **I32), torch.full((B * Hkv + 16,), 7, **I32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.bd_paged_select(*a, 16, budget, lists=lists[:-16].view(B, Hkv, budget), lens=lens[:-16].view(B, Hkv), workspace=ws[:n],
                             stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (ws[n:] == 255).all() and (lists[-16:] == 7).all() and (lens[-16:] == 7).all()
    _replayed(lambda: bd.bd_paged_select(*a, 16, budget, workspace=ws[:n]), f"select, form {form}", [
        lambda: None, lambda: a[3].mul_(2).clamp_(max=400), lambda: a[3].copy_(a[3].flip(0)), lambda: a[0].mul_(-1),
        lambda: a[1].add_(0.25), lambda: ws.fill_(255)])


def test_choice_with_absent_pages():
    """Pages outside the pool are not chosen, whatever their place: all, the first and last ones, or all but fewer than the budget."""
    P, width = 16, 50
    q, s, table, lens = _select_inputs(4, 4, 2, 128, 1, P, width, [800, 790, 33, 800], 8)
    table[0, ::2] = -1
    table[1, 0] = 1 << 30
    table[1, 49] = -(1 << 31)
    table[2, :] = s.shape[0]
    table[3, 3:] = -1
    for budget, first, last in ((8, 1, 2), (3, 0, 3), (40, 2, 2)):
        _select_check(q, s, table, lens, P, budget, first, last, f"absent budget{budget}")


def test_choice_by_the_last_bits():
    """Scores that differ in their last float64 bits alone, far below float32's."""
    P, width, D = 16, 64, 64
    q = torch.zeros((1, 1, 1, D), dtype=BF, device=DEV)
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -20
    s = torch.zeros((width, 1, 2, D), dtype=BF, device=DEV)
    s[:, 0, :, 0] = 128.0
    s[:, 0, :, 1] = (torch.arange(width, device=DEV) * 37 % 64).float()[:, None] * 2.0 ** -20
    _select_check(q, s, torch.arange(width, **I32)[None].contiguous(), _ints([width * P]), P, 9, 0, 0, "last bits")


def test_choice_replayed_and_on_another_stream():
    a = _select_inputs(3, 8, 2, 64, 4, 16, 40, [640, 100, 333], 12)
    want = bd.bd_paged_select(*a, 16, 8)
    ws = torch.full((bd.bd_paged_select_workspace_bytes(3, 4, 8, 2, 64, 16, 40, 8),), 255, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.bd_paged_select(*a, 16, 8, workspace=ws, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    _replayed(lambda: bd.bd_paged_select(*a, 16, 8), "select", [
        lambda: None, lambda: a[3].copy_(_ints([1, 640, 0])), lambda: a[0].mul_(-1), lambda: a[1].add_(0.25)])


# ---------------------------------------------------------------------------
# decoding over lists

def _check_sparse(a, got, tag, scale=None):
    q, kp, vp, lists, lens, kn, vn = a
    fixed = (lists.tolist(), lens.tolist())
    want = oracle.sparse_decode_forward(_np(q), _np(kp), _np(vp), *fixed, _np(kn), _np(vn), scale)
    size = oracle.sparse_decode_forward(_np(q), _np(kp), np.abs(_np(vp)), *fixed, _np(kn), None if vn is None else np.abs(_np(vn)),
                                        scale)
    _check(got, want, size[0], tag)


def _sparse_inputs(B, Hq, Hkv, D, S, P, K, hi, order, block, seed):
    g = torch.Generator().manual_seed(seed)
    n = K + 40
    kp, vp = _cache(n, Hkv, P, D, order, g)
    lists = torch.stack([torch.randperm(n, generator=g)[:K] for _ in range(B * Hkv)]).view(B, Hkv, K).to(torch.int32).to(DEV)
    lens = torch.randint(0, hi + 1, (B, Hkv), generator=g, dtype=torch.int32).to(DEV)
    q = (torch.randn((B, Hq, S, D), generator=g) * 0.5).to(BF).to(DEV)
    new = [(torch.randn((B, Hkv, S, D), generator=g) * 0.5).to(BF).to(DEV) if block else None for _ in range(2)]
    return [q, kp, vp, lists, lens, *new]


@pytest.mark.parametrize("B,Hq,Hkv,D,S,P,K,hi,order,block", [
    (1, 1, 1, 64, 1, 16, 1, 16, "heads", False), (1, 32, 8, 128, 1, 16, 32, 512, "heads", False),
    (3, 8, 2, 64, 4, 64, 5, 320, "tokens", True), (2, 12, 3, 128, 1, 16, 20, 300, "sides", False),
    (2, 33, 1, 64, 1, 16, 9, 144, "heads", False), (2, 8, 4, 64, 32, 32, 8, 256, "tokens", True),
    (3, 8, 2, 128, 32, 32, 13, 416, "heads", True), (2, 4, 2, 64, 36, 16, 7, 100, "heads", False),
    (2, 4, 1, 128, 64, 128, 3, 384, "tokens", True), (150, 4, 2, 128, 1, 16, 4, 64, "heads", False),
    (5, 8, 8, 128, 1, 1024, 2, 2048, "tokens", False), (4, 4, 2, 64, 2, 16, 6, 0, "heads", False),
])
def test_sparse_decode_matches_oracle(B, Hq, Hkv, D, S, P, K, hi, order, block):
    print(f"[sparse] lists B{B} H{Hq}/{Hkv} D{D} S{S} P{P} K{K} {order} block={block}", flush=True)
    a = _sparse_inputs(B, Hq, Hkv, D, S, P, K, hi, order, block, B + K)
    _check_sparse(a, bd.bd_attn_paged_sparse_decode_fwd(*a), f"lists K{K} S{S}")


def test_sparse_absent_pages_clamped_lengths_and_scale():
    a = _sparse_inputs(3, 8, 2, 64, 4, 16, 9, 144, "heads", True, 23)
    a[3][0, 0, 2:4] = -1
    a[3][0, 1, :] = 1 << 30
    a[3][1, 0, 0] = a[1].shape[0]
    a[4].copy_(_ints([[144, 140], [1000, -3], [7, 1 << 30]]))
    _check_sparse(a, bd.bd_attn_paged_sparse_decode_fwd(*a, scale=0.2), "absent", 0.2)
    _check_sparse(a[:5] + [None, None], bd.bd_attn_paged_sparse_decode_fwd(*a[:5]), "absent, cache alone")


def test_sparse_reads_nothing_else_and_replays():
    a = _sparse_inputs(3, 8, 2, 128, 1, 16, 9, 144, "tokens", False, 29)
    want = bd.bd_attn_paged_sparse_decode_fwd(*a)
    keep = torch.zeros(a[1].shape[0], 2, 16, dtype=torch.bool)
    ids, lens = a[3].cpu(), a[4].tolist()
    for b in range(3):
        for h in range(2):
            for j in range(lens[b][h]):
                keep[ids[b, h, j // 16], h, j % 16] = True
            ids[b, h, -(-lens[b][h] // 16):] = (1 << 31) - 1
    a[3].copy_(ids)
    for x in a[1:3]:
        x.copy_(torch.where(keep.to(DEV)[..., None], x, float("nan")))
    ws = torch.full((bd.bd_attn_paged_sparse_decode_workspace_bytes(3, 1, 8, 2, 128, 16, 9),), 255, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bd.bd_attn_paged_sparse_decode_fwd(*a, workspace=ws, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    fewer = [a[4].clone(), (a[4] // 2).to(torch.int32), a[4] * 0]
    _replayed(lambda: bd.bd_attn_paged_sparse_decode_fwd(*a), "lists", [lambda x=x: a[4].copy_(x) for x in fewer])


# ---------------------------------------------------------------------------
# together

def test_rollout_over_chosen_pages():
    """Blocks of tokens into a paged cache (plan, write), their pages summarised, pages chosen and decoded over: each
    step against the oracle, and a budget that holds every page against decoding over the whole cache."""
    B, Hq, Hkv, D, S, P, width = 3, 8, 2, 64, 8, 16, 12
    g = torch.Generator(device=DEV).manual_seed(31)
    pages = B * width + 4
    kp, vp = (torch.full((pages, Hkv, P, D), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    s = torch.full((pages, Hkv, 2, D), float("nan"), dtype=BF, device=DEV)
    free = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table, lens, head = torch.full((B, width), -1, **I32), _ints([0, 0, 0]), _ints([0])
    rope, w = bd.bd_rope_table(width * P, D, device=DEV), torch.ones(D, dtype=BF, device=DEV)
    for step in range(20):
        new = _ints([8, 8 if step % 3 else 5, 0 if step == 4 else 8])
        plan = bd.bd_paged_plan(lens, new, table, free, head, pages, P, S=S)
        assert plan.state[1] == 0
        x = torch.randn((B, S, (Hq + 2 * Hkv) * D), generator=g, device=DEV).to(BF).unflatten(-1, (-1, D))
        q = bd.bd_qk_norm_rope_paged(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], w, w, rope, plan.positions,
                                     plan.slots, kp, vp) * 0.25
        bd.bd_paged_summarize(kp, table, lens, plan.lens, s)
        lens, head = plan.lens, plan.state[:1]
        if step % 5 < 3:
            continue
        keys, n = _np(kp), lens.tolist()
        for b in range(B):
            for j in range(-(-n[b] // P)):
                k = keys[int(table[b, j]), :, :min(P, n[b] - j * P)]
                assert (_np(s[int(table[b, j])]) == np.stack([k.min(1), k.max(1)], 1)).all()
        clean = torch.nan_to_num(s)
        chosen = _select_check(q, clean, table, lens, P, 4, 1, 1, f"step {step}")
        assert all(torch.equal(a, b) for a, b in zip(chosen, bd.bd_paged_select(q, s, table, lens, P, 4, 1, 1)))
        got = bd.bd_attn_paged_sparse_decode_fwd(q, kp, vp, *chosen)
        _check_sparse([q, torch.nan_to_num(kp), torch.nan_to_num(vp), *chosen, None, None], got, f"rollout {step}")
        every = bd.bd_paged_select(q, s, table, lens, P, width, 1, 1)
        assert (every.lens == lens[:, None]).all()
        a, b = bd.bd_attn_paged_sparse_decode_fwd(q, kp, vp, *every), bd.bd_attn_paged_decode_fwd(q, kp, vp, table, lens)
        # (two roundings of the same value, and sums in other orders)
        assert ((a[0].float() - b[0].float()).abs() <= 2.0 ** -7 * b[0].float().abs() + 2 * SUMS * 4).all()
        assert ((a[1] - b[1]).abs() <= 2 * SUMS).all()


def test_rollout_of_samples_of_two_prompts():
    """Prompts written once each, five answers from them (three and two): block by block, decoding with the shared
    prefix against the oracle and against decoding over tables that repeat the prefix's pages."""
    Hq, Hkv, D, S, P, width = 8, 4, 128, 4, 16, 6
    g = torch.Generator(device=DEV).manual_seed(37)
    prompts, sizes, B = [48, 37], [3, 2], 5
    pages = 60
    kp, vp = (torch.zeros((pages, Hkv, P, D), dtype=BF, device=DEV) for _ in range(2))
    free = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    rope, w = bd.bd_rope_table(256, D, device=DEV), torch.ones(D, dtype=BF, device=DEV)

    def write(n, positions, slots):
        x = torch.randn((*n, (Hq + 2 * Hkv) * D), generator=g, device=DEV).to(BF).unflatten(-1, (-1, D))
        return bd.bd_qk_norm_rope_paged(x[..., :Hq, :], x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :], w, w, rope, positions, slots,
                                        kp, vp)

    prefix_table = torch.full((2, width), -1, **I32)
    plan = bd.bd_paged_plan(_ints([0, 0]), _ints(prompts), prefix_table, free, _ints([0]), pages, P, total=sum(prompts))
    write((sum(prompts),), plan.positions, plan.slots)
    prefix_lens, head = plan.lens, plan.state[:1]
    table, lens = torch.full((B, width), -1, **I32), torch.zeros(B, **I32)
    behind = torch.repeat_interleave(prefix_lens, _ints(sizes).long())[:, None]
    for step in range(6):
        plan = bd.bd_paged_plan(lens, torch.full((B,), S, **I32), table, free, head, pages, P, S=S)
        q = write((B, S), plan.positions + behind, plan.slots) * 0.25
        lens, head = plan.lens, plan.state[:1]
        a = [q, kp, vp, _ints(sizes), prefix_table, prefix_lens, table, lens, None, None]
        got = bd.bd_attn_paged_shared_decode_fwd(*a)
        _check_shared(a, got, f"samples {step}")
        # the first prompt fills its pages: its answers' tables may repeat them
        joined = torch.cat([prefix_table[0, :3].expand(3, 3), table[:3]], 1).contiguous()
        want = bd.bd_attn_paged_decode_fwd(q[:3], kp, vp, joined, lens[:3] + 48)
        assert ((got[0][:3].float() - want[0].float()).abs() <= 2.0 ** -7 * want[0].float().abs() + 2 * SUMS * 4).all()
        assert ((got[1][:3] - want[1]).abs() <= 2 * SUMS).all()
