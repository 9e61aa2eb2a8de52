"""Plain fp64 decoding for sequences that share prefixes, page summaries, the choice
of pages and decoding over lists of pages (definitions of include/bd_attn.h,
bd_attn_paged_shared_decode_fwd, bd_paged_summarize, bd_paged_select and
bd_attn_paged_sparse_decode_fwd)."""
from __future__ import annotations

import numpy as np


def _keys(pages, ids, n, g):
    """Rows below n of KV head g in the pages `ids`, those outside the pool left out: [.., D]."""
    P = pages.shape[2]
    rows = [pages[ids[j // P], g, j % P] for j in range(min(max(int(n), 0), len(ids) * P)) if 0 <= ids[j // P] < len(pages)]
    return np.array(rows).reshape(-1, pages.shape[3])


def _attend(q, k, v, scale):
    """One head's rows q [S, D] over keys k, v: (o [S, D], lse [S]); nothing seen: 0 and -inf."""
    if len(k) == 0:
        return np.zeros(q.shape), np.full(len(q), -np.inf)
    z = q @ k.T * scale
    m = z.max(axis=1)
    e = np.exp(z - m[:, None])
    return e @ v / e.sum(axis=1)[:, None], m + np.log(e.sum(axis=1))


def shared_decode_forward(Q, Kp, Vp, sizes, prefix_table, prefix_lens, table, lens, Kn=None, Vn=None, scale=None):
    """-> (O [B,Hq,S,D], LSE [B,Hq,S]) in float64."""
    Q, Kp, Vp = (np.asarray(t, dtype=np.float64) for t in (Q, Kp, Vp))
    B, Hq, S, D = Q.shape
    Hkv = Kp.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    group = [g for g, n in enumerate(sizes) for _ in range(min(max(int(n), 0), B))][:B]
    group += [None] * (B - len(group))
    O, LSE = np.zeros(Q.shape), np.zeros(Q.shape[:3])
    for g in range(Hkv):
        shared = {}
        for b in range(B):
            kv = []
            for i, (pages, new) in enumerate(((Kp, Kn), (Vp, Vn))):
                x = [_keys(pages, table[b], lens[b], g)]
                if group[b] is not None:
                    at = (group[b], i)
                    if at not in shared:
                        shared[at] = _keys(pages, prefix_table[group[b]], prefix_lens[group[b]], g)
                    x.insert(0, shared[at])
                if new is not None:
                    x.append(np.asarray(new[b, g], dtype=np.float64))
                kv.append(np.concatenate(x))
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                O[b, h], LSE[b, h] = _attend(Q[b, h], *kv, scale)
    return O, LSE


def summarize(Kp, table, before, lens, summaries):
    """-> summaries [pages, Hkv, 2, D], those of the sequences' new pages over their keys."""
    out = np.array(summaries)
    pages, _, P, _ = Kp.shape
    for b in range(len(lens)):
        n = min(max(int(lens[b]), 0), len(table[b]) * P)
        if before[b] >= n:  # no new position
            continue
        for j in range(max(int(before[b]), 0) // P, -(-n // P)):
            if 0 <= table[b][j] < pages:
                k = Kp[table[b][j], :, :min(P, n - j * P)]
                out[table[b][j]] = np.stack([k.min(axis=1), k.max(axis=1)], axis=1)
    return out


def page_scores(Q, summaries, ids):
    """[rows of a KV head, D] and [pages, 2, D] of that head -> scores of the pages, row by row as defined."""
    lo, hi = summaries[ids, 0], summaries[ids, 1]
    return sum(np.maximum(q * lo, q * hi).sum(axis=1) for q in Q)


def select(Q, summaries, table, lens, P, budget, first, last):
    """-> (lists [B,Hkv,budget], keys in them [B,Hkv])."""
    Q, summaries = (np.asarray(t, dtype=np.float64) for t in (Q, summaries))
    B, Hq, S, D = Q.shape
    Hkv = summaries.shape[1]
    lists, keys = np.full((B, Hkv, budget), -1), np.zeros((B, Hkv), dtype=np.int64)
    for b in range(B):
        n = min(max(int(lens[b]), 0), len(table[b]) * P)
        used = -(-n // P)
        real = [j for j in range(used) if 0 <= table[b][j] < len(summaries)]
        kept = [j for j in real if j < first or j >= used - last]
        for g in range(Hkv):
            rows = Q[b, g * (Hq // Hkv):(g + 1) * (Hq // Hkv)].reshape(-1, D)
            score = dict(zip(real, page_scores(rows, summaries[:, g], [table[b][j] for j in real]))) if real else {}
            rest = sorted((j for j in real if j not in kept), key=lambda j: (-score[j], j))
            chosen = sorted(kept + rest[:budget - len(kept)])
            lists[b, g, :len(chosen)] = [table[b][j] for j in chosen]
            keys[b, g] = sum(min(P, n - j * P) for j in chosen)
    return lists, keys


def sparse_decode_forward(Q, Kp, Vp, lists, list_lens, Kn=None, Vn=None, scale=None):
    """-> (O [B,Hq,S,D], LSE [B,Hq,S]) in float64."""
    Q, Kp, Vp = (np.asarray(t, dtype=np.float64) for t in (Q, Kp, Vp))
    B, Hq, S, D = Q.shape
    G = Hq // Kp.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    O, LSE = np.zeros(Q.shape), np.zeros(Q.shape[:3])
    for b in range(B):
        for h in range(Hq):
            k, v = (_keys(c, lists[b][h // G], list_lens[b][h // G], h // G) for c in (Kp, Vp))
            if Kn is not None:
                k, v = (np.concatenate([x, np.asarray(n[b, h // G], dtype=np.float64)]) for x, n in ((k, Kn), (v, Vn)))
            O[b, h], LSE[b, h] = _attend(Q[b, h], k, v, scale)
    return O, LSE
