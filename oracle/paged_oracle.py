"""Plain fp64 decoding over a paged KV cache, and page tables built sequence by
sequence (definitions of include/bd_attn.h, bd_attn_paged_decode_fwd and
bd_paged_plan)."""
from __future__ import annotations

import numpy as np


def paged_decode_forward(Q, Kp, Vp, table, lens, Kn=None, Vn=None, scale=None):
    """Q [B,Hq,S,D], Kp/Vp [pages,Hkv,P,D], table [B,width] -> (O [B,Hq,S,D], LSE [B,Hq,S]) in float64."""
    Q, Kp, Vp = (np.asarray(t, dtype=np.float64) for t in (Q, Kp, Vp))
    B, Hq, S, D = Q.shape
    pages, Hkv, P, _ = Kp.shape
    width = table.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    O, LSE = np.zeros(Q.shape), np.full(Q.shape[:3], -np.inf)
    for b in range(B):
        at = np.arange(min(max(int(lens[b]), 0), width * P))
        ids = np.asarray(table)[b, at // P]
        seen = (ids >= 0) & (ids < pages)
        ids, rows = ids[seen], at[seen] % P
        for h in range(Hq):
            g = h // (Hq // Hkv)
            k, v = Kp[ids, g, rows], Vp[ids, g, rows]
            if Kn is not None:
                k = np.concatenate([k, np.asarray(Kn[b, g], dtype=np.float64)])
                v = np.concatenate([v, np.asarray(Vn[b, g], dtype=np.float64)])
            if len(k) == 0:
                continue
            z = Q[b, h] @ k.T * scale
            m = z.max(axis=1, keepdims=True)
            e = np.exp(z - m)
            LSE[b, h] = (m + np.log(e.sum(axis=1, keepdims=True)))[:, 0]
            O[b, h] = e @ v / e.sum(axis=1, keepdims=True)
    return O, LSE


def paged_plan(lens, new, table, free, head, num_pages, P, S=0, total=0):
    """-> (table, lens, cu, slots, positions, state): int lists and arrays, one token after another."""
    table = np.array(table)
    B, width = table.shape
    cap = width * P
    head = min(max(int(head), 0), len(free))
    count = B * S if S else total
    slots, positions = np.full(count, -1), np.zeros(count, dtype=np.int64)
    out, cu, at, lost = [], [0], 0, 0
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        m = max(int(new[b]), 0)
        m = min(m, S) if S else m
        end = min(n + m, cap)
        for j in range(-(-n // P), -(-end // P)):  # pages begun by this call
            page = int(free[head]) if head < len(free) else -1
            head = min(head + 1, len(free))
            table[b, j] = page if 0 <= page < num_pages else -1
        for i in range(m):
            t = b * S + i if S else at + i
            page = table[b, (n + i) // P] if n + i < cap else -1
            ok = 0 <= page < num_pages
            lost += not (ok and t < count)
            if t < count:
                positions[t] = n + i
                slots[t] = page * P + (n + i) % P if ok else -1
        at += m
        out.append(end)
        cu.append(at)
    return table, np.array(out), np.array(cu), slots, positions, np.array([head, lost])
