"""GPU parity of the paged cache: page tables and slots, writing into pages, and
decoding over them, each against the fp64 oracle, and a rollout of all three.

Decoding's tolerances are those of the dense decode tests, whose arithmetic it
shares (bf16 operands and probabilities, float32 accumulation): O max-abs <= 2e-2
and rel-L2 <= 5e-3, LSE max-abs <= 1e-3.  Plans are integers and have to be equal.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_22234_amd as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16
O_MAX, O_REL, LSE_MAX = 2e-2, 5e-3, 1e-3


def _qkv_views(qkv, Hq, Hkv, D):
    return qkv.unflatten(-1, (Hq + 2 * Hkv, D)).split([Hq, Hkv, Hkv], dim=-2)


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _check(o, lse, want, tag):
    O, L, (Or, Lr) = _np(o), _np(lse), want
    seen = np.isfinite(Lr)
    assert (np.isneginf(L) == ~seen).all() and (O[~seen] == 0).all()
    e = dict(o_max=float(np.abs(O - Or).max()), lse_max=float(np.abs(L[seen] - Lr[seen]).max(initial=0.0)),
             o_rel=float(np.linalg.norm(O - Or) / max(np.linalg.norm(Or), 1e-30)))
    print(f"[paged] {tag} errors {e}", flush=True)
    assert e["o_max"] <= O_MAX and e["o_rel"] <= O_REL and e["lse_max"] <= LSE_MAX, e


def _pages(n, Hkv, P, D, order, g, fill=None):
    """k_pages, v_pages [n, Hkv, P, D] in one of the memory orders."""
    def rows(*shape):
        if fill is not None:
            return torch.full(shape, fill, dtype=BF, device=DEV)
        return (torch.randn(shape, generator=g) * 0.5).to(BF).to(DEV)

    if order == "heads":
        return rows(n, Hkv, P, D), rows(n, Hkv, P, D)
    if order == "tokens":
        return tuple(rows(n, P, Hkv, D).permute(0, 2, 1, 3) for _ in range(2))
    if order == "outer":                      # [heads, pages, rows, D]
        return tuple(rows(Hkv, n, P, D).permute(1, 0, 2, 3) for _ in range(2))
    if order == "pairs":                      # [pages, 2, heads, rows, D]
        kv = rows(n, 2, Hkv, P, D)
        return kv[:, 0], kv[:, 1]
    kv = rows(n, P, Hkv, 2, D).permute(3, 0, 2, 1, 4)   # K and V of a head side by side
    return kv[0], kv[1]


def _inputs(B, Hq, Hkv, D, S, P, width, lens, order, seed, block, spare=3):
    g = torch.Generator().manual_seed(seed)
    need = [-(-min(max(n, 0), width * P) // P) for n in lens]
    n = max(1, sum(need) + spare)
    kp, vp = _pages(n, Hkv, P, D, order, g)
    ids = torch.randperm(n, generator=g, dtype=torch.int64).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    q = (torch.randn((B, Hq, S, D), generator=g) * 0.5).to(BF).to(DEV)
    new = [(torch.randn((B, Hkv, S, D), generator=g) * 0.5).to(BF).to(DEV) if block else None for _ in range(2)]
    return q, kp, vp, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), *new


def _oracle(q, kp, vp, table, lens, kn=None, vn=None, scale=None):
    return oracle.paged_decode_forward(_np(q), _np(kp), _np(vp), table.cpu().numpy(), lens.cpu().numpy(), _np(kn), _np(vn),
                                       scale)


# Query rows per KV head (G*S) at the edges of the wave and team sizes, page
# sizes below, at and above the key tiles, lengths around pages and tiles, all orders.
DECODE = [
    # B, Hq, Hkv, D, S, P, width, lens, order, block
    (1, 1, 1, 64, 1, 16, 1, [1], "heads", False),
    (4, 32, 8, 128, 1, 16, 40, [1, 15, 16, 640], "tokens", False),
    (3, 8, 2, 128, 1, 32, 20, [0, 33, 640], "pairs", False),            # a row without keys
    (2, 4, 4, 64, 1, 128, 5, [127, 513], "sides", False),
    (5, 32, 8, 128, 4, 64, 20, [0, 1, 63, 65, 1280], "heads", True),
    (3, 4, 2, 64, 4, 1024, 2, [0, 1024, 1025], "heads", True),
    (2, 33, 1, 64, 1, 16, 9, [129, 64], "tokens", False),               # 33 rows: two waves
    (3, 4, 2, 128, 32, 16, 50, [700, 0, 33], "heads", True),            # 64 rows
    (2, 65, 1, 64, 1, 32, 10, [257, 1], "pairs", False),                # 65 rows: four waves
    (6, 8, 2, 128, 32, 32, 13, [400, 0, 1, 31, 32, 97], "tokens", True),  # 128 rows
    (2, 8, 2, 64, 36, 16, 13, [191, 65], "heads", True),                # 144 rows: two groups
    (2, 4, 1, 128, 64, 64, 3, [150, 3], "sides", True),                 # 256 rows: two groups
    (2, 4, 1, 128, 64, 64, 3, [150, 0], "heads", False),                # ... and a sequence without keys
    (300, 4, 2, 64, 2, 16, 4, [i % 65 for i in range(300)], "tokens", True),
    (300, 2, 1, 128, 1, 16, 4, [i % 3 * 30 for i in range(300)], "heads", False),
    (16, 4, 4, 128, 1, 256, 47, [12000, 3] * 8, "heads", False),        # runs cross items
    (3, 8, 4, 64, 3, 1 << 15, 2, [40000, 0, 32768], "outer", True),     # the largest pages, heads outermost
    (2, 32, 1, 64, 40, 16, 20, [300, 7], "outer", True),                # 1280 rows: ten groups
    (5, 4, 2, 128, 1, 16, 2, [0, 0, 0, 0, 0], "heads", False),          # no key at all
    (2, 12, 3, 64, 16, 64, 30, [1900, 1023], "tokens", True),           # 64 rows at D = 64
]


@pytest.mark.parametrize("B,Hq,Hkv,D,S,P,width,lens,order,block", DECODE)
def test_decode_matches_oracle(B, Hq, Hkv, D, S, P, width, lens, order, block):
    print(f"[paged] B{B} H{Hq}/{Hkv} D{D} S{S} P{P} width{width} {order} block={block} lens={lens[:6]}", flush=True)
    a = _inputs(B, Hq, Hkv, D, S, P, width, lens, order, seed=B * S + P, block=block)
    o, lse = bd.bd_attn_paged_decode_fwd(*a)
    _check(o, lse, _oracle(*a), f"P{P} S{S}")


@pytest.mark.parametrize("S,P,Hq,D", [(1, 16, 8, 128), (4, 64, 8, 128), (32, 16, 4, 128), (32, 32, 8, 128), (1, 16, 8, 64),
                                      (16, 16, 8, 64), (32, 64, 8, 64)])
@pytest.mark.parametrize("block", [False, True])
def test_pages_that_are_none(S, P, Hq, D, block):
    """Entries outside the pool, singly and in runs: their keys are left out; a
    sequence whose pages are all none sees its own block or nothing."""
    B, Hkv, width = 4, 2, 300 // P + 2
    a = list(_inputs(B, Hq, Hkv, D, S, P, width, [300, 299, 150, 33], "heads", 77 + S, block))
    t = a[3]
    t[0, 1] = -1
    t[0, 3 % (300 // P)] = 1 << 30
    t[1, : 256 // P] = a[1].shape[0]                        # first id past the pool
    t[2, : -(-150 // P)] = -(1 << 31)                       # none at all
    o, lse = bd.bd_attn_paged_decode_fwd(*a)
    _check(o, lse, _oracle(*a), f"absent S{S} P{P}")


def test_lengths_are_clamped_and_scale_given():
    B, Hq, Hkv, D, S, P, width = 3, 4, 2, 64, 1, 16, 3
    a = list(_inputs(B, Hq, Hkv, D, S, P, width, [48, 48, 48], "heads", 5, False))
    a[4] = torch.tensor([1000, -7, 1 << 30], dtype=torch.int32, device=DEV)
    o, lse = bd.bd_attn_paged_decode_fwd(*a, scale=0.3)
    _check(o, lse, _oracle(*a, scale=0.3), "clamped")


@pytest.mark.parametrize("S,P,order", [(1, 16, "heads"), (1, 64, "tokens"), (32, 16, "tokens"), (16, 32, "pairs")])
def test_nothing_else_is_read(S, P, order):
    """Rows of the pages past a length, pages of no sequence, and table entries
    past it hold NaN and wild ids: the result's bits stay."""
    B, Hq, Hkv, D, width = 3, 8, 2, 128, 9
    lens = [70, 131, 1]
    q, kp, vp, table, cl, kn, vn = _inputs(B, Hq, Hkv, D, S, P, width, lens, order, 6, S > 1)
    want = bd.bd_attn_paged_decode_fwd(q, kp, vp, table, cl, kn, vn)
    keep = torch.zeros(kp.shape[0], P, dtype=torch.bool)
    t = table.cpu()
    for b, n in enumerate(lens):
        n = min(n, width * P)
        for j in range(n):
            keep[t[b, j // P], j % P] = True
        t[b, -(-n // P):] = (1 << 31) - 1
    for x in (kp, vp):
        x.copy_(torch.where(keep.to(DEV)[:, None, :, None], x, float("nan")))
    got = bd.bd_attn_paged_decode_fwd(q, kp, vp, t.to(DEV), cl, kn, vn)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_strided_table_shared_pages_and_determinism():
    """Table rows inside a wider array; two sequences on the same pages; the same bits
    twice, on another stream, and without the other sequences but for rounding."""
    a = list(_inputs(4, 16, 4, 128, 1, 16, 20, [300, 300, 17, 255], "heads", 8, False))
    a[3][1] = a[3][0]
    a[0][1] = a[0][0]
    wide = torch.full((4, 33), 1 << 20, dtype=torch.int32, device=DEV)
    wide[:, 5:25] = a[3]
    want = bd.bd_attn_paged_decode_fwd(*a)
    _check(*want, _oracle(*a), "shared")
    assert float((want[0][0].float() - want[0][1].float()).abs().max()) <= 1e-2
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [bd.bd_attn_paged_decode_fwd(*a[:3], wide[:, 5:25], *a[4:]), bd.bd_attn_paged_decode_fwd(*a),
           bd.bd_attn_paged_decode_fwd(*a, stream=side)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))


@pytest.mark.parametrize("D,S,lens", [(128, 1, [1500]), (64, 4, [700, 33, 0, 2000]), (128, 8, [300, 4000])])
def test_one_wave_rounds_the_result_only(D, S, lens):
    """Up to 32 query rows per KV head P enters with 16 bits: O is off by the rounding of the
    result, at most 2^-8 of each value, and by P's, 2^-17 of the sum of |p v|, with float32 sums
    below that (at most 2^-15 of it in all)."""
    a = _inputs(len(lens), 16, 4, D, S, 32, 130, lens, "heads", 31 + D, S > 1)
    o, _ = bd.bd_attn_paged_decode_fwd(*a)
    want, _ = _oracle(*a)
    size, _ = oracle.paged_decode_forward(_np(a[0]), _np(a[1]), np.abs(_np(a[2])), a[3].cpu().numpy(), a[4].cpu().numpy(),
                                          _np(a[5]), None if a[6] is None else np.abs(_np(a[6])))
    err = np.abs(_np(o) - want)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * size
    print(f"[paged] one wave D{D} S{S}: largest error / tolerance {float((err / (tol + 1e-30)).max()):.3f}", flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("D,S,lens", [(128, 16, [700, 33]), (64, 16, [1, 1000]), (128, 32, [40, 1500]), (64, 32, [600, 0, 97]),
                                      (128, 64, [150, 900])])
@pytest.mark.parametrize("block", [False, True])
def test_teams_round_the_result_only(D, S, lens, block):
    """The same with more rows per KV head (64, 128, and 256 in two groups): P has 16 bits there too."""
    a = _inputs(len(lens), 8, 2, D, S, 32, 60, lens, "heads", 57 + D + S, block)
    o, _ = bd.bd_attn_paged_decode_fwd(*a)
    want, _ = _oracle(*a)
    size, _ = oracle.paged_decode_forward(_np(a[0]), _np(a[1]), np.abs(_np(a[2])), a[3].cpu().numpy(), a[4].cpu().numpy(),
                                          _np(a[5]), None if a[6] is None else np.abs(_np(a[6])))
    err = np.abs(_np(o) - want)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * size
    print(f"[paged] teams D{D} S{S} block={block}: largest error / tolerance {float((err / (tol + 1e-30)).max()):.3f}", flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("B", [16000, 16500])
def test_many_tiles_on_shared_pages(B):
    """Just below and above 2^22 key tiles (sequences of 1024 tokens on the same
    pages, 8 heads): the runs' cuts in 32 and in 64 bits.  Equal queries give equal
    results but for where the runs cut them: float32 sums, P rounded to bf16."""
    H, D, P, n = 8, 64, 64, 1024
    g = torch.Generator().manual_seed(4)
    kp, vp = _pages(n // P, H, P, D, "heads", g)
    q = (torch.randn((1, H, 1, D), generator=g) * 0.5).to(BF).to(DEV).repeat(B, 1, 1, 1)
    table = torch.randperm(n // P, generator=g).to(torch.int32).to(DEV).repeat(B, 1)
    lens = torch.full((B,), n, dtype=torch.int32, device=DEV)
    o, lse = bd.bd_attn_paged_decode_fwd(q, kp, vp, table, lens)
    _check(o[:1], lse[:1], _oracle(q[:1], kp, vp, table[:1], lens[:1]), "many tiles")
    assert float((o.float() - o[:1].float()).abs().max()) <= 1e-2 and float((lse - lse[:1]).abs().max()) <= 1e-4


def test_runs_of_a_long_call():
    """25,600 key tiles at D = 128 (as many runs as the grid holds), rows of pages shared by the sequences."""
    B, Hq, Hkv, D, P = 400, 16, 8, 128, 32
    g = torch.Generator().manual_seed(5)
    kp, vp = _pages(40, Hkv, P, D, "tokens", g)
    q = (torch.randn((B, Hq, 1, D), generator=g) * 0.5).to(BF).to(DEV)
    table = torch.randint(0, 40, (B, 8), generator=g, dtype=torch.int32).to(DEV)
    lens = torch.randint(240, 257, (B,), generator=g, dtype=torch.int32).to(DEV)
    o, lse = bd.bd_attn_paged_decode_fwd(q, kp, vp, table, lens)
    pick = [0, 1, 133, 266, 399]
    _check(o[pick], lse[pick], _oracle(q[pick], kp, vp, table[pick], lens[pick]), "long call")


def test_offsets_past_32_bits():
    """Pages behind 2^32 bytes and 2^31 elements of an 8 GiB array."""
    B, Hq, Hkv, D, P, n = 2, 8, 8, 128, 64, 66000
    kp = torch.empty((n, Hkv, P, D), dtype=BF, device=DEV)
    assert kp.numel() > 1 << 32
    vp = torch.empty_like(kp)
    ids = torch.tensor([[n - 1, 5, n - 2, 32768], [32767, n - 3, 16384, 40000]], dtype=torch.int32, device=DEV)
    for x in (kp, vp):
        x[ids.long().view(-1)] = (torch.randn((8, Hkv, P, D), device=DEV) * 0.5).to(BF)
    q = (torch.randn((B, Hq, 1, D), device=DEV) * 0.5).to(BF)
    lens = torch.tensor([250, 256], dtype=torch.int32, device=DEV)
    o, lse = bd.bd_attn_paged_decode_fwd(q, kp, vp, ids, lens)
    small = [x[ids.long().view(-1)] for x in (kp, vp)]
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4)
    _check(o, lse, _oracle(q, *small, table, lens), "far pages")
    # ... and written there
    rope = bd.bd_rope_table(300, D, device=DEV)
    w = torch.ones(D, dtype=BF, device=DEV)
    x = torch.randn((1, 2, Hkv, D), device=DEV).to(BF)
    slots = torch.tensor([[(n - 1) * P + 63, 40000 * P]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([[3, 4]], dtype=torch.int32, device=DEV)
    bd.bd_qk_norm_rope_paged(x, x, x, w, w, rope, pos, slots, kp, vp)
    _, ko, vo = bd.bd_qk_norm_rope_fwd(x, x, x, w, w, rope, pos)
    for pages, y in ((kp, ko), (vp, vo)):
        assert torch.equal(pages[n - 1, :, 63], y[0, :, 0]) and torch.equal(pages[40000, :, 0], y[0, :, 1])


# ---------------------------------------------------------------------------
# page tables and slots

def _plan_check(lens, new, table, free, head, pages, P, S=None, total=None):
    t = torch.tensor(table, dtype=torch.int32, device=DEV)
    dev = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, new, free, [head])]
    p = bd.bd_paged_plan(dev[0], dev[1], t, dev[2], dev[3], pages, P, S=S, total=total)
    want = oracle.paged_plan(lens, new, table, free, head, pages, P, S or 0, total or 0)
    for name, a, b in zip(("table", "lens", "cu", "slots", "positions", "state"), (t, *p), want):
        np.testing.assert_array_equal(a.cpu().numpy().reshape(np.shape(b)), b, err_msg=name)
    return p


@pytest.mark.parametrize("B,P,width,S,hi", [
    (1, 16, 4, 1, 60), (1, 16, 4, None, 60), (7, 64, 10, 4, 600), (64, 16, 64, None, 500), (255, 16, 9, 3, 140),
    (256, 32, 9, None, 140), (257, 16, 9, 1, 140), (1000, 16, 30, None, 90), (5000, 16, 3, 2, 47), (3, 1024, 6, None, 5000),
    (1 << 16, 16, 2, 1, 31), (2, 1 << 15, 8, None, 200000),
])
def test_plan_matches_oracle(B, P, width, S, hi):
    rng = np.random.default_rng(B + P)
    lens = rng.integers(0, hi + 1, B)
    new = rng.integers(0, (S or max(2, hi // 2)) + 1, B)
    new[rng.random(B) < 0.2] = 0
    need = int((-(-np.minimum(lens, width * P) // P)).sum())
    pages = need + B * (2 + (S or hi // 2) // P) + 9
    ids = rng.permutation(pages)
    table = np.full((B, width), -1)
    at = 0
    for b in range(B):
        k = -(-min(int(lens[b]), width * P) // P)
        table[b, :k] = ids[at:at + k]
        at += k
    print(f"[plan] B{B} P{P} S{S}", flush=True)
    _plan_check(lens, new, table, ids[at:], 3, pages, P, S, int(new.sum()) + 5)


def test_plan_edges():
    """Full rows, a free list that runs out or is empty, wild lengths, ids and head, and no new tokens."""
    P, width = 16, 3
    table = np.array([[4, 5, 6], [7, -1, -1], [-1, -1, -1], [9, 99, -1], [-3, -1, -1]])
    free = [10, 11, 12, 13, 14]
    for S, total in ((20, None), (None, 70)):
        _plan_check([48, 3, 0, 20, 5], [4, 20, 0, 3, 6], table, free, 0, 30, P, S, total)      # rows full, pages that are none
        _plan_check([40, 3, 0, 16, 0], [20, 20, 14, 3, 0], table, free, 3, 30, P, S, total)    # runs out in the middle
        _plan_check([40, 3, 0, 16, 0], [20, 13, 2, 16, 1], table, free, 99, 30, P, S, total)   # head past the end
        _plan_check([1000, -5, 0, 2, 1], [5, -3, 20, 0, 0], table, free, -2, 30, P, S, total)  # clamped
        _plan_check([0, 0, 0, 0, 0], [0, 0, 0, 0, 0], table, free, 0, 30, P, S, total)
        _plan_check([0, 3, 0, 16, 0], [1, 13, 2, 16, 1], table, [], 0, 30, P, S, total)


def test_plan_ids_outside_the_pool():
    """A free list's id outside the pool: entered as -1, its tokens without a slot."""
    p = torch.tensor
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.full((2, 3), -1, **i32)
    plan = bd.bd_paged_plan(p([0, 0], **i32), p([20, 4], **i32), table, p([1, 50, -4, 2], **i32), p([0], **i32), 8, 16, S=20)
    assert table.tolist() == [[1, -1, -1], [-1, -1, -1]]
    assert plan.slots[0].tolist() == list(range(16, 32)) + [-1] * 4 and (plan.slots[1] == -1).all()
    assert plan.positions[1].tolist() == [0, 1, 2, 3] + [0] * 16 and plan.state[0] == 3


def test_plan_too_small_a_total():
    """Tokens past total are dropped without a write past the arrays, and reported."""
    i32 = dict(dtype=torch.int32, device=DEV)
    buf = torch.full((40,), 77, **i32)
    table = torch.full((2, 4), -1, **i32)
    plan = bd.bd_paged_plan(torch.zeros(2, **i32), torch.tensor([10, 1 << 30], **i32), table,
                            torch.arange(8, **i32), torch.zeros(1, **i32), 8, 16, total=12, slots=buf[:12],
                            positions=buf[16:28])
    assert (buf[12:16] == 77).all() and (buf[28:] == 77).all()
    assert plan.slots.tolist() == list(range(10)) + [16, 17] and int(plan.state[1]) > 0


def _damaged(B, P, width, pages, seed, bad):
    """Lengths, new lengths, a table of stale ids and a free list with a share of ids outside the pool."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, width * P + 1, B)
    new = rng.integers(0, 3 * P, B) * (rng.random(B) < 0.8)
    table = rng.integers(0, pages, (B, width))
    free = np.where(rng.random(2 * B) < bad, rng.choice([-1, -(1 << 31), pages, (1 << 31) - 1], 2 * B), rng.permutation(2 * B) % pages)
    return lens, new, table, free


@pytest.mark.parametrize("S", [20, None])
def test_plan_counts_the_tokens_of_ids_outside_the_pool(S):
    """state[1] is exact where the free list holds ids outside the pool: in a whole page, the
    last one of a sequence, several in a row, and behind a list that runs out."""
    total = None if S else 70
    _plan_check([0, 0], [20, 4], np.full((2, 3), -1), [1, 50, -4, 2], 0, 8, 16, S, total)
    table = np.array([[4, 5, 6], [7, 3, 3], [3, 3, 3], [3, 9, 3]])
    _plan_check([0, 3, 0, 32], [17, 20, 0, 7], table, [8, 8, 1, 99], 0, 8, 16, S, total)
    _plan_check([0, 3, 0, 32], [17, 20, 0, 7], table, [0, -9, 8], 1, 8, 16, S, total)
    for B in (40, 700):
        lens, new, table, free = _damaged(B, 16, 5, 900, B, 0.3)
        _plan_check(lens, new, table, free, 3, 900, 16, S, None if S else int(new.sum()) + 5)


@pytest.mark.parametrize("B", [3, 40, 700])
@pytest.mark.parametrize("share", [0.0, 0.01, 0.4, 0.97])
def test_plan_enters_the_pages_of_tokens_past_total(B, share):
    """Packed tokens that sum to more than total: those past it get no slot and are counted once,
    and every page that is taken from the list is entered, over the stale ids of the table."""
    for bad in (0.0, 0.3):
        lens, new, table, free = _damaged(B, 16, 5, 900, B, bad)
        new[:2] = [40, 90]
        lens[:2] = [3, 0]
        for total in (int(new.sum() * share), int(new[0]) + 37):
            _plan_check(lens, new, table, free, 1, 900, 16, None, total)
        _plan_check(lens, new, table, free, len(free) - 5, 900, 16, None, int(new.sum() * share))


def test_plan_of_more_pages_than_an_int_counts():
    """40 sequences that would need 2^26 pages each: the list gives what it has, the head stays inside it."""
    i32 = dict(dtype=torch.int32, device=DEV)
    width = 1 << 26  # (rows of 2^30 tokens; a row's entries are written for the tokens below total alone)
    table = torch.empty((40, width), **i32)
    table[0, 0] = -1
    plan = bd.bd_paged_plan(torch.zeros(40, **i32), torch.full((40,), 1 << 30, **i32), table, torch.arange(8, **i32),
                            torch.tensor([3], **i32), 8, 16, total=4)
    assert int(table[0, 0]) == 3 and plan.slots.tolist() == [48, 49, 50, 51]
    assert plan.lens.tolist() == [1 << 30] * 40 and plan.cu.tolist() == [0, 1 << 30] + [2**31 - 1] * 39
    assert plan.state.tolist() == [8, 2**31 - 1]


# ---------------------------------------------------------------------------
# writing into pages

@pytest.mark.parametrize("order", ["heads", "tokens", "pairs", "sides", "outer"])
@pytest.mark.parametrize("B,N,Hq,Hkv,D,P", [(1, 1, 1, 1, 64, 16), (5, 4, 8, 2, 128, 64), (1, 333, 16, 4, 128, 16)])
def test_write_into_pages(order, B, N, Hq, Hkv, D, P):
    """Keys and values of the plain call at their slots, bitwise; every other row stays."""
    g = torch.Generator().manual_seed(N + D)
    T = B * N
    n = -(-T // P) + 2
    kp, vp = _pages(n, Hkv, P, D, order, g)
    before = kp.clone(), vp.clone()
    qkv = torch.randn((B, N, (Hq + 2 * Hkv) * D), generator=g).to(BF).to(DEV)
    q, k, v = _qkv_views(qkv, Hq, Hkv, D)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(DEV) for _ in range(2)]
    rope = bd.bd_rope_table(100, D, device=DEV)
    pos = torch.randint(0, 100, (B, N), generator=g, dtype=torch.int32).to(DEV)
    slots = torch.randperm(n * P, generator=g)[:T].to(torch.int32)
    if T > 3:
        slots[1], slots[2], slots[T - 1] = -1, n * P, 1 << 30      # outside the pages: not written
    slots = slots.view(B, N).to(DEV)
    qo = bd.bd_qk_norm_rope_paged(q, k, v, *w, rope, pos, slots, kp, vp)
    want = bd.bd_qk_norm_rope_fwd(q, k, v, *w, rope, pos)
    assert torch.equal(qo, want[0])
    at = slots.view(-1).long()
    ok = (at >= 0) & (at < n * P)
    for pages, old, x in zip((kp, vp), before, want[1:]):
        rows = old.permute(0, 2, 1, 3).reshape(n * P, Hkv, D)
        rows[at[ok]] = x.transpose(1, 2).reshape(T, Hkv, D)[ok]
        assert torch.equal(pages, rows.view(n, P, Hkv, D).permute(0, 2, 1, 3))


# ---------------------------------------------------------------------------
# a rollout

class _Rollout:
    """Plan, write, attend: the calls a program makes, on buffers of its own."""

    def __init__(self, B, Hq, Hkv, D, P, width, S, order):
        g = torch.Generator().manual_seed(99)
        self.pages = B * width
        self.dims = B, Hq, Hkv, D, P, S
        self.kp, self.vp = _pages(self.pages, Hkv, P, D, order, g, fill=0.0)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table = torch.full((B, width), -1, **i32)
        self.free = torch.randperm(self.pages, generator=g).to(torch.int32).to(DEV)
        self.lens, self.head = torch.zeros(B, **i32), torch.zeros(1, **i32)
        self.w = [(1 + 0.2 * torch.randn(D, generator=g)).to(BF).to(DEV) for _ in range(2)]
        self.rope = bd.bd_rope_table(width * P, D, device=DEV)

    def step(self, qkv, new, S=None, total=None):
        """The next tokens: their attention over everything cached, themselves included."""
        B, Hq, Hkv, D, P, _ = self.dims
        plan = bd.bd_paged_plan(self.lens, new, self.table, self.free, self.head, self.pages, P, S=S, total=total)
        q = bd.bd_qk_norm_rope_paged(*_qkv_views(qkv, Hq, Hkv, D), *self.w, self.rope, plan.positions, plan.slots,
                                     self.kp, self.vp)
        return plan, q

    def take(self, plan):
        self.lens.copy_(plan.lens)
        self.head.copy_(plan.state[:1])


@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_rollout_of_tokens_and_blocks(order):
    """Prompts of different lengths go in packed, then single tokens, then a block
    denoised twice over the cache; each step against the oracle on keys kept by hand."""
    B, Hq, Hkv, D, P, width = 4, 8, 2, 64, 16, 8
    r = _Rollout(B, Hq, Hkv, D, P, width, 1, order)
    g = torch.Generator().manual_seed(1)
    w, table = [_np(x) for x in r.w], _np(r.rope)
    keys = [np.zeros((Hkv, 0, D)) for _ in range(B)]
    vals = [np.zeros((Hkv, 0, D)) for _ in range(B)]

    def project(*lead):
        return torch.randn((*lead, (Hq + 2 * Hkv) * D), generator=g).to(BF).to(DEV)

    def bf(x):
        return _np(torch.from_numpy(x).to(BF))

    def keep(b, qkv, pos):
        _, k, v = _qkv_views(qkv, Hq, Hkv, D)
        keys[b] = np.concatenate([keys[b], bf(oracle.norm_rope(_np(k), w[1], table, pos, 1e-6))], axis=1)
        vals[b] = np.concatenate([vals[b], _np(v).swapaxes(0, 1)], axis=1)

    def want(b, qn, kn=None, vn=None):
        k, v = keys[b], vals[b]
        if kn is not None:
            k, v = np.concatenate([k, kn], 1), np.concatenate([v, vn], 1)
        n = np.array([k.shape[1]])
        pad = width * P + 64
        kk, vv = (np.concatenate([x, np.zeros((Hkv, pad - x.shape[1], D))], 1)[None] for x in (k, v))
        return oracle.paged_decode_forward(qn[None], kk, vv, np.array([[0]]), n)

    # prompts (one of them empty), packed
    lens = [37, 0, 5, 64]
    i32 = dict(dtype=torch.int32, device=DEV)
    qkv = project(sum(lens))
    plan, _ = r.step(qkv, torch.tensor(lens, **i32), total=sum(lens))
    r.take(plan)
    at = 0
    for b, n in enumerate(lens):
        keep(b, qkv[at:at + n], np.arange(n))
        at += n
    # single tokens: the new one's key is in the cache when it attends
    for _ in range(3):
        qkv = project(B, 1)
        pos = r.lens.cpu().numpy().copy()
        plan, q = r.step(qkv, torch.ones(B, **i32), S=1)
        r.take(plan)
        o, lse = bd.bd_attn_paged_decode_fwd(q, r.kp, r.vp, r.table, r.lens)
        for b in range(B):
            keep(b, qkv[b], pos[b:b + 1])
            _check(o[b:b + 1], lse[b:b + 1], want(b, _np(q[b])), f"token of {b}")
    # a block of 4: denoised against the cache, then written into it (not for a sequence that is done)
    S = 4
    pos = r.lens[:, None] + torch.arange(S, **i32)
    for _ in range(2):
        qkv = project(B, S)
        q, kn, vn = bd.bd_qk_norm_rope_fwd(*_qkv_views(qkv, Hq, Hkv, D), *r.w, r.rope, pos)
        o, lse = bd.bd_attn_paged_decode_fwd(q, r.kp, r.vp, r.table, r.lens, kn, vn)
        for b in range(B):
            _check(o[b:b + 1], lse[b:b + 1], want(b, _np(q[b]), _np(kn[b]), _np(vn[b])), f"block of {b}")
    new = torch.tensor([S, S, 0, S], **i32)
    plan, q = r.step(qkv, new, S=S)
    assert torch.equal(plan.positions[[0, 1, 3]], pos[[0, 1, 3]].to(torch.int32)) and (plan.slots[2] == -1).all()
    r.take(plan)
    for b in (0, 1, 3):
        keep(b, qkv[b], pos[b].cpu().numpy())
    o, lse = bd.bd_attn_paged_decode_fwd(q, r.kp, r.vp, r.table, r.lens)
    for b in range(B):
        _check(o[b:b + 1], lse[b:b + 1], want(b, _np(q[b])), f"cached block of {b}")
    assert int(plan.state[1]) == 0


def test_captured_step_follows_the_lengths():
    """One token step of a batch captured as a graph and replayed: tables, slots and
    lengths move on the device alone; a second rollout runs the same calls eagerly."""
    B, Hq, Hkv, D, P, width = 3, 8, 2, 128, 16, 6
    runs = [_Rollout(B, Hq, Hkv, D, P, width, 1, "heads") for _ in range(2)]
    qkv = torch.zeros((B, 1, (Hq + 2 * Hkv) * D), dtype=BF, device=DEV)
    ones = torch.ones(B, dtype=torch.int32, device=DEV)

    def step(r):
        plan, q = r.step(qkv, ones, S=1)
        r.take(plan)
        return bd.bd_attn_paged_decode_fwd(q, r.kp, r.vp, r.table, r.lens)

    step(runs[1])                               # loads the kernels
    runs[1] = _Rollout(B, Hq, Hkv, D, P, width, 1, "heads")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(runs[0])
    for i in range(40):
        qkv.normal_()
        graph.replay()
        want = step(runs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
        for name in ("kp", "vp", "table", "lens", "head"):
            assert torch.equal(getattr(runs[0], name), getattr(runs[1], name)), (i, name)
    assert runs[0].lens.tolist() == [40] * B
