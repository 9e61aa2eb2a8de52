"""Measured calls of rollouts that share a prompt, and of rollouts over long contexts of which
each step reads a part, both over a paged KV cache.

- decoding of sequences in groups that share a prefix (several samples of one prompt), the
  prefix's keys and values read once for the group;
- summaries of pages (smallest and largest value of each key feature), kept as pages fill;
- pages chosen for each sequence and KV head by an upper bound of their scores;
- decoding over the chosen pages alone.

`own` selects the library's entry points; otherwise the same is computed with elementary
torch operations in float32, and the scores that pages are ordered by in float64.  Heads,
head sizes, block sizes and lengths are those of paper_2512_22234_amd/workloads.py and of the
tests, with odd and ragged sizes between them.  Inputs are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BF16 = torch.bfloat16


# ---------------------------------------------------------------------------
# the cases

def listed():
    return [
        # eight samples of one prompt, the first tokens of their answers: latency
        dict(name="shared_single", kind="shared", groups=1, n=8, S=1, block=False, Hq=32, Hkv=8, D=128, P=16,
             plo=1500, phi=1500, lo=1, hi=200, lens=21, order="heads"),
        # a rollout batch, eight samples of each prompt, token by token; token-major pages
        dict(name="shared_tokens", kind="shared", groups=16, n=8, S=1, block=False, Hq=32, Hkv=8, D=128, P=16,
             plo=512, phi=8192, lo=16, hi=2048, lens=22, order="tokens"),
        # the same in blocks of 4, groups of uneven size
        dict(name="shared_blocks", kind="shared", groups=8, n=9, S=4, block=True, Hq=32, Hkv=8, D=128, P=64,
             plo=1024, phi=8192, lo=16, hi=1000, lens=23, order="heads"),
        # blocks of 32 tokens behind long prompts, many rows for each key
        dict(name="shared_block32", kind="shared", groups=3, n=8, S=32, block=True, Hq=32, Hkv=8, D=128, P=32,
             plo=4096, phi=8192, lo=16, hi=1000, lens=24, order="heads"),
        # the pages that a finished block of every sequence lies in
        dict(name="summarize_block", kind="summarize", B=64, Hkv=8, D=128, P=64, S=4, lo=512, hi=8000, lens=25,
             order="heads"),
        # the pages of a batch of new prompts, token-major
        dict(name="summarize_prompts", kind="summarize", B=40, Hkv=8, D=128, P=16, S=0, lo=100, hi=4000, lens=26,
             order="tokens"),
        # interactive use: the next token of one sequence
        dict(name="select_single", kind="select", B=1, S=1, Hq=32, Hkv=8, D=128, P=16, lo=1500, hi=1500, budget=32,
             first=1, last=2, lens=27),
        # the next block of a rollout batch at mixed points of its generation
        dict(name="select_blocks", kind="select", B=64, S=4, Hq=32, Hkv=8, D=128, P=16, lo=512, hi=8192, budget=64,
             first=1, last=2, lens=28),
        # two long documents, blocks of 32
        dict(name="select_long", kind="select", B=2, S=32, Hq=32, Hkv=8, D=128, P=64, lo=120000, hi=131072, budget=64,
             first=1, last=4, lens=29),
        # one token of one sequence over 32 chosen pages: latency
        dict(name="sparse_single", kind="sparse", B=1, S=1, block=False, Hq=32, Hkv=8, D=128, P=16, budget=32, held=94,
             lo=500, hi=512, lens=30, order="heads"),
        # the next token of a rollout batch, 64 chosen pages of 16 a KV head
        dict(name="sparse_tokens", kind="sparse", B=128, S=1, block=False, Hq=32, Hkv=8, D=128, P=16, budget=64,
             held=160, lo=512, hi=1024, lens=31, order="tokens"),
        # blocks of 32 tokens, chosen pages of 32
        dict(name="sparse_block32", kind="sparse", B=24, S=32, block=True, Hq=32, Hkv=8, D=128, P=32, budget=64,
             held=128, lo=200, hi=2048, lens=32, order="heads"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


HEADS = [(32, 8), (16, 4), (16, 8), (12, 4), (8, 8)]


def draw(rng):
    """One more case of the ranges above (no more work than the largest)."""
    kind = rng.choice(["shared", "shared", "shared", "summarize", "select", "select", "sparse", "sparse"])
    Hq, Hkv = rng.choice(HEADS)
    D = rng.choice([64, 128, 128])
    P = rng.choice([16, 32, 64, 128])
    order = rng.choice(["heads", "tokens"])
    lens = rng.randrange(1 << 20)
    if kind == "shared":
        block = rng.random() < 0.6
        S = rng.choice([1, 4, 8, 16, 32]) if block else 1
        groups = _log_int(rng, 1, 16 if S <= 8 else 3)
        plo = _log_int(rng, 64, 4096)
        lo = _log_int(rng, 1, 500)
        return dict(kind=kind, groups=groups, n=rng.randint(1, 8), S=S, block=block, Hq=Hq, Hkv=Hkv, D=D, P=P,
                    plo=plo, phi=_log_int(rng, plo, 8192), lo=lo, hi=_log_int(rng, lo, 1000), lens=lens, order=order)
    if kind == "summarize":
        lo = _log_int(rng, 16, 1000)
        return dict(kind=kind, B=_log_int(rng, 1, 40), Hkv=Hkv, D=D, P=P, S=rng.choice([0, 1, 4, 16, 32]), lo=lo,
                    hi=_log_int(rng, lo, 4000), lens=lens, order=order)
    if kind == "select":
        B = _log_int(rng, 1, 64)
        top = 8192 if B > 4 else 131072
        lo = _log_int(rng, 64, top // 4)
        return dict(kind=kind, B=B, S=rng.choice([1, 4, 8, 16, 32]), Hq=Hq, Hkv=Hkv, D=D, P=P, lo=lo,
                    hi=_log_int(rng, lo, top), budget=_log_int(rng, 6, 128), first=rng.randint(0, 2),
                    last=rng.randint(0, 4), lens=lens)
    block = rng.random() < 0.5
    S = rng.choice([1, 4, 8, 16, 32]) if block else 1
    budget = _log_int(rng, 1, 2048 // P)
    lo = _log_int(rng, 1, budget * P)
    B = _log_int(rng, 1, 128 if S == 1 else 24)
    return dict(kind=kind, B=B, S=S, block=block, Hq=Hq, Hkv=Hkv, D=D, P=P, budget=budget,
                held=_log_int(rng, budget, 2 * budget), lo=lo, hi=_log_int(rng, lo, budget * P), lens=lens, order=order)


# ---------------------------------------------------------------------------
# inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _log_lens(rng, lo, hi, n):
    return [int(round(lo * (hi / lo) ** x)) for x in rng.random(n)]


def _case_lens(case):
    """The case's lengths, log-uniform: shared (group sizes, prefixes, own keys), sparse (rows of each
    list), summarize (tokens before, tokens after), select (tokens)."""
    rng = np.random.default_rng(case["lens"])
    kind = case["kind"]
    if kind == "shared":
        gr, n = case["groups"], case["n"]
        sizes = rng.integers(max(1, n - 2), n + 1, gr).tolist() if gr > 1 else [n]
        return sizes, _log_lens(rng, case["plo"], case["phi"], gr), _log_lens(rng, case["lo"], case["hi"], sum(sizes))
    if kind == "sparse":
        return _log_lens(rng, case["lo"], case["hi"], case["B"] * case["Hkv"])
    lens = _log_lens(rng, case["lo"], case["hi"], case["B"])
    if kind == "summarize":
        return [n if case["S"] else 0 for n in lens], [n + case["S"] for n in lens]
    return lens


def _pages(n, P):
    return -(-n // P)


def _tables(lists, P, g):
    """Page tables with random distinct pages: lists of lengths -> (int32 tables, -1 past each length; pages in use)."""
    total = sum(_pages(n, P) for lens in lists for n in lens)
    ids = torch.randperm(total + 5, generator=g, device=DEV).to(torch.int32).cpu()
    at, out = 0, []
    for lens in lists:
        t = torch.full((len(lens), max(_pages(n, P) for n in lens) + 1), -1, dtype=torch.int32)
        for b, n in enumerate(lens):
            k = _pages(n, P)
            t[b, :k] = ids[at:at + k]
            at += k
        out.append(t.to(DEV))
    return out, total + 5


def _cache(shape, order, g):
    """bf16 pages [pages, Hkv, P, D], with the heads or the tokens of a page outermost in memory."""
    n, H, P, D = shape
    if order == "heads":
        return torch.randn((n, H, P, D), generator=g, device=DEV, dtype=BF16) * 0.5
    return (torch.randn((n, P, H, D), generator=g, device=DEV, dtype=BF16) * 0.5).permute(0, 2, 1, 3)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    kind = case["kind"]
    g = _generator(seed)
    st = dict(case=case)
    Hkv, D, P = case["Hkv"], case["D"], case["P"]
    if kind == "shared":
        sizes, prefix, lens = _case_lens(case)
        (st["prefix_table"], st["table"]), total = _tables([prefix, lens], P, g)
        st.update(sizes=_int32(sizes), prefix_lens=_int32(prefix), lens=_int32(lens))
        B = len(lens)
    elif kind == "summarize":
        before, after = _case_lens(case)
        (st["table"],), total = _tables([after], P, g)
        st.update(before=_int32(before), lens=_int32(after))
    elif kind == "select":
        B, lens = case["B"], _case_lens(case)
        (st["table"],), total = _tables([lens], P, g)
        st["lens"] = _int32(lens)
    else:
        # a sequence holds pages of its own, of which each KV head has some, in the order of their positions
        B, K, held = case["B"], case["budget"], case["held"]
        rows, total = _case_lens(case), B * held + 5
        pages = torch.randperm(total, generator=g, device=DEV)[:B * held].view(B, 1, held).expand(B, Hkv, held)
        some = torch.rand((B, Hkv, held), generator=g, device=DEV).topk(K, dim=2)[1].sort(2)[0]
        used = _int32([_pages(n, P) for n in rows]).view(B, Hkv, 1)
        lists = torch.where(torch.arange(K, device=DEV) < used, torch.gather(pages, 2, some), -1)
        st.update(lists=lists.to(torch.int32), rows=_int32(rows).view(B, Hkv))
    if kind == "select":
        # summaries of keys around a mean of each page's own
        st["summaries"] = torch.empty((total, Hkv, 2, D), dtype=BF16, device=DEV)
        for a in range(0, total, 4096):
            n = min(4096, total - a)
            k = torch.randn((n, Hkv, P, D), generator=g, device=DEV, dtype=BF16) * 0.4
            k += torch.randn((n, Hkv, 1, D), generator=g, device=DEV, dtype=BF16) * 0.3
            st["summaries"][a:a + n, :, 0] = k.amin(2)
            st["summaries"][a:a + n, :, 1] = k.amax(2)
    else:
        st["kp"] = _cache((total, Hkv, P, D), case["order"], g)
    if kind == "summarize":
        st["summaries"] = torch.zeros((total, Hkv, 2, D), dtype=BF16, device=DEV)
        return st
    S, Hq = case["S"], case["Hq"]
    st["q"] = torch.randn((B, Hq, S, D), generator=g, device=DEV, dtype=BF16) * 0.5
    if kind != "select":
        st["vp"] = _cache((total, Hkv, P, D), case["order"], g)
        for name in ("kn", "vn"):
            st[name] = (torch.randn((B, Hkv, S, D), generator=g, device=DEV, dtype=BF16) * 0.5
                        if case["block"] else None)
    return st


# ---------------------------------------------------------------------------
# one pass

def run(st):
    if own:
        return _run_own(st)
    with torch.no_grad():
        return _plain[st["case"]["kind"]](st)


def _run_own(st):
    import paper_2512_22234_amd as bd
    case = st["case"]
    kind = case["kind"]
    if kind == "shared":
        return bd.bd_attn_paged_shared_decode_fwd(st["q"], st["kp"], st["vp"], st["sizes"], st["prefix_table"],
                                                  st["prefix_lens"], st["table"], st["lens"], st["kn"], st["vn"])
    if kind == "summarize":
        return bd.bd_paged_summarize(st["kp"], st["table"], st["before"], st["lens"], st["summaries"])
    if kind == "select":
        return bd.bd_paged_select(st["q"], st["summaries"], st["table"], st["lens"], case["P"], case["budget"],
                                  first=case["first"], last=case["last"])
    return bd.bd_attn_paged_sparse_decode_fwd(st["q"], st["kp"], st["vp"], st["lists"], st["rows"], st["kn"], st["vn"])


def _attend(q, k, v, seen):
    """Masked softmax attention in float32: q [N, R, D], k, v [N, keys, D], seen [N, keys] -> (o, lse)."""
    x = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(q.shape[-1]))
    x.masked_fill_(~seen[:, None, :], -math.inf)
    top = x.max(-1, keepdim=True)[0]
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    return torch.matmul(x, v) / total, (top + total.log())[..., 0]


def _gathered(pages, ids):
    """Rows of the pages ids [N, width] of each KV head: float32 [N, Hkv, width * P, D]."""
    n, H, P, D = pages.shape
    return pages[ids].permute(0, 2, 1, 3, 4).reshape(ids.shape[0], H, -1, D).float()


def _below(table, P, lens):
    """Which rows of the pages in each table row hold keys: [N, width * P]."""
    return torch.arange(table.shape[1] * P, device=DEV)[None, :] < lens[:, None]


def _shaped(case, o, lse, B):
    S, Hq, D = case["S"], case["Hq"], case["D"]
    return o.reshape(B, Hq, S, D).to(BF16), lse.reshape(B, Hq, S)


def _plain_shared(st):
    case = st["case"]
    Hq, Hkv, D, P, S = (case[x] for x in ("Hq", "Hkv", "D", "P", "S"))
    B = st["lens"].shape[0]
    group = torch.repeat_interleave(torch.arange(case["groups"], device=DEV), st["sizes"].long(), output_size=B)
    ids = torch.cat([st["prefix_table"][group], st["table"]], 1).long().clamp(min=0)
    k, v = _gathered(st["kp"], ids), _gathered(st["vp"], ids)
    seen = torch.cat([_below(st["prefix_table"], P, st["prefix_lens"])[group], _below(st["table"], P, st["lens"])], 1)
    if st["kn"] is not None:
        k, v = torch.cat([k, st["kn"].float()], 2), torch.cat([v, st["vn"].float()], 2)
        seen = torch.cat([seen, seen.new_ones((B, S))], 1)
    n = k.shape[2]
    o, lse = _attend(st["q"].float().reshape(B * Hkv, -1, D), k.reshape(B * Hkv, n, D), v.reshape(B * Hkv, n, D),
                     seen[:, None, :].expand(B, Hkv, n).reshape(B * Hkv, n))
    return _shaped(case, o, lse, B)


def _plain_summarize(st):
    P = st["case"]["P"]
    table, before, lens = st["table"].long(), st["before"].long(), st["lens"].long()
    j = torch.arange(table.shape[1], device=DEV)
    b, j = torch.nonzero((j[None, :] >= before[:, None] // P) & (j[None, :] * P < lens[:, None]), as_tuple=True)
    ids = table[b, j]
    rows = st["kp"][ids].float()
    seen = (j[:, None] * P + torch.arange(P, device=DEV)[None, :] < lens[b][:, None])[:, None, :, None]
    lo = torch.where(seen, rows, math.inf).amin(2)
    hi = torch.where(seen, rows, -math.inf).amax(2)
    st["summaries"][ids] = torch.stack([lo, hi], 2).to(BF16)
    return st["summaries"]


def _plain_select(st):
    case = st["case"]
    B, Hkv, D, P, K = (case[x] for x in ("B", "Hkv", "D", "P", "budget"))
    table, lens = st["table"].long(), st["lens"].long()
    width = table.shape[1]
    q = st["q"].double().view(B, Hkv, -1, D)
    up, down = q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)
    s = st["summaries"][table.clamp(min=0)].permute(0, 2, 1, 3, 4)
    scores = (s[..., 0, :].double() * down[:, :, None]).sum(-1) + (s[..., 1, :].double() * up[:, :, None]).sum(-1)
    j = torch.arange(width, device=DEV)[None, :]
    used = (lens + P - 1)[:, None] // P
    kept = (j < case["first"]) | (j >= used - case["last"])
    scores = torch.where(kept[:, None, :], math.inf, scores)
    scores = torch.where((j < used)[:, None, :], scores, -math.inf)
    # the highest scores, equal ones by position, then all in the order of their positions
    at = torch.sort(scores, dim=2, descending=True, stable=True)[1][:, :, :K]
    at = torch.where(torch.gather(scores, 2, at) > -math.inf, at, width).sort(2)[0]
    if at.shape[2] < K:
        at = torch.cat([at, at.new_full((B, Hkv, K - at.shape[2]), width)], 2)
    some = at < width
    ids = torch.gather(table[:, None, :].expand(B, Hkv, width), 2, at.clamp(max=width - 1))
    tail = (at == used[:, None, :] - 1).any(2)
    rows = some.sum(2) * P - torch.where(tail, used * P - lens[:, None], 0)
    return torch.where(some, ids, -1).to(torch.int32), rows.to(torch.int32)


def _plain_sparse(st):
    case = st["case"]
    B, S, Hkv, D, P, K = (case[x] for x in ("B", "S", "Hkv", "D", "P", "budget"))
    ids = st["lists"].long().clamp(min=0)
    head = torch.arange(Hkv, device=DEV)[None, :, None].expand(B, Hkv, K)
    k, v = (c[ids, head].reshape(B * Hkv, K * P, D).float() for c in (st["kp"], st["vp"]))
    seen = torch.arange(K * P, device=DEV)[None, :] < st["rows"].view(-1, 1)
    if st["kn"] is not None:
        k = torch.cat([k, st["kn"].float().view(B * Hkv, S, D)], 1)
        v = torch.cat([v, st["vn"].float().view(B * Hkv, S, D)], 1)
        seen = torch.cat([seen, seen.new_ones((B * Hkv, S))], 1)
    o, lse = _attend(st["q"].float().reshape(B * Hkv, -1, D), k, v, seen)
    return _shaped(case, o, lse, B)


_plain = dict(shared=_plain_shared, summarize=_plain_summarize, select=_plain_select, sparse=_plain_sparse)


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    kind, Hkv, D, P = case["kind"], case["Hkv"], case["D"], case["P"]
    if kind == "summarize":
        before, after = _case_lens(case)
        pages = sum(_pages(n, P) - m // P for m, n in zip(before, after))
        rows = sum(n - m // P * P for m, n in zip(before, after))
        return {"bytes": rows * Hkv * D * 2 + pages * (Hkv * D * 4 + 4) + 8 * case["B"], "flops": rows * Hkv * D * 2}
    Hq, S = case["Hq"], case["S"]
    if kind == "select":
        pages = sum(_pages(n, P) for n in _case_lens(case))
        B, K = case["B"], case["budget"]
        return {"bytes": pages * (Hkv * D * 4 + 4) + B * Hq * S * D * 2 + B * Hkv * (K * 4 + 4) + 4 * B,
                "flops": pages * Hkv * D * 4 + B * Hq * S * D * 2}
    if kind == "shared":
        sizes, prefix, lens = _case_lens(case)
        B = len(lens)
        block = B * S if case["block"] else 0
        keys = sum(prefix) + sum(lens) + block
        pairs = sum(n * p for n, p in zip(sizes, prefix)) + sum(lens) + block
        entries = sum(_pages(n, P) for n in prefix + lens)
        return {"bytes": keys * Hkv * D * 4 + 4 * entries + B * Hq * S * (D * 4 + 4), "flops": pairs * Hq * S * D * 4}
    rows, B = _case_lens(case), case["B"]
    keys = sum(rows) + (B * Hkv * S if case["block"] else 0)
    return {"bytes": keys * D * 4 + 4 * sum(_pages(n, P) for n in rows) + B * Hq * S * (D * 4 + 4),
            "flops": keys * (Hq // Hkv) * S * D * 4}


# ---------------------------------------------------------------------------
# the same in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return dict(shared=_exact_shared, summarize=_exact_summarize, select=_exact_select,
                sparse=_exact_sparse)[case["kind"]](st)


def _rows(pages, ids, n, head=slice(None)):
    """The first n rows in the pages `ids`, of every KV head or of one: float64 [.., n, D]."""
    x = pages[ids[:_pages(n, pages.shape[2])].long()][:, head].double()
    return x.transpose(-4, -3).flatten(-3, -2)[..., :n, :] if x.dim() == 4 else x.flatten(0, 1)[:n]


def _softmax_sum(q, k, v):
    """Definition: q [.., R, D], k, v [.., keys, D] -> (o, lse)."""
    z = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
    return torch.matmul(torch.softmax(z, dim=-1), v), torch.logsumexp(z, dim=-1)


def _exact_shared(st):
    case = st["case"]
    sizes, prefix, lens = _case_lens(case)
    S, Hq, Hkv, D = (case[x] for x in ("S", "Hq", "Hkv", "D"))
    o = torch.empty((len(lens), Hq, S, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((len(lens), Hq, S), dtype=torch.float64, device=DEV)
    b = 0
    for g, (n, p) in enumerate(zip(sizes, prefix)):
        shared = [_rows(c, st["prefix_table"][g], p) for c in (st["kp"], st["vp"])]
        for _ in range(n):
            kv = []
            for x, c, new in zip(shared, (st["kp"], st["vp"]), (st["kn"], st["vn"])):
                kv.append(torch.cat([x, _rows(c, st["table"][b], lens[b])] + ([] if new is None else [new[b].double()]), 1))
            ob, lb = _softmax_sum(st["q"][b].double().view(Hkv, -1, D), *kv)
            o[b], lse[b] = ob.view(Hq, S, D), lb.view(Hq, S)
            b += 1
    return o, lse


def _exact_summarize(st):
    before, after = _case_lens(st["case"])
    P, out = st["case"]["P"], st["summaries"].double()
    for b, (m, n) in enumerate(zip(before, after)):
        a = m // P
        ids = st["table"][b, a:_pages(n, P)].long()
        k = st["kp"][ids].double()
        out[ids, :, 0], out[ids, :, 1] = k.amin(2), k.amax(2)
        tail = n - (_pages(n, P) - 1) * P
        out[ids[-1], :, 0], out[ids[-1], :, 1] = k[-1, :, :tail].amin(1), k[-1, :, :tail].amax(1)
    return out


def _exact_select(st):
    return None  # whole numbers: equal or wrong


def _exact_sparse(st):
    case = st["case"]
    B, S, Hq, Hkv, D = (case[x] for x in ("B", "S", "Hq", "Hkv", "D"))
    o = torch.empty((B, Hkv, Hq // Hkv * S, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, Hkv, Hq // Hkv * S), dtype=torch.float64, device=DEV)
    q, rows = st["q"].view(o.shape), st["rows"].tolist()
    for b in range(B):
        for h in range(Hkv):
            k, v = (_rows(c, st["lists"][b, h], rows[b][h], h) for c in (st["kp"], st["vp"]))
            if st["kn"] is not None:
                k, v = torch.cat([k, st["kn"][b, h].double()]), torch.cat([v, st["vn"][b, h].double()])
            o[b, h], lse[b, h] = _softmax_sum(q[b, h].double(), k, v)
    return o.view(B, Hq, S, D), lse.view(B, Hq, S)
