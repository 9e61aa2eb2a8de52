"""Plain fp64 norms of queries and keys with the rotary embedding, and their
gradients (formulas of include/bd_attn.h, bd_qk_norm_rope_fwd / _bwd)."""
from __future__ import annotations

import numpy as np


def rope_table(n: int, D: int, theta: float = 1e6, inv_freq=None) -> np.ndarray:
    """[n, D]: cos(p f_j), then sin(p f_j), f_j = theta^(-2j/D) or inv_freq[j]."""
    if inv_freq is None:
        inv_freq = float(theta) ** (-2.0 * np.arange(D // 2) / D)
    a = np.arange(n, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None, :]
    return np.concatenate([np.cos(a), np.sin(a)], axis=1)


def _angles(rope, pos, D):
    """cos and sin [.., N, 1, D/2] for positions clamped to the table."""
    cs = np.asarray(rope, dtype=np.float64)[np.clip(pos, 0, len(rope) - 1)][..., None, :]
    return cs[..., :D // 2], cs[..., D // 2:]


def norm_rope(x, w, rope, pos, eps: float):
    """x [.., N, H, D] -> normalised, rotated heads [.., H, N, D]; pos [.., N]."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    D = x.shape[-1]
    c, s = _angles(rope, pos, D)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y1, y2 = y[..., :D // 2], y[..., D // 2:]
    return np.swapaxes(np.concatenate([y1 * c - y2 * s, y2 * c + y1 * s], axis=-1), -3, -2)


def norm_rope_backward(d, x, w, rope, pos, eps: float):
    """Gradients for d [.., H, N, D]: dx [.., N, H, D], dw [D], and sum |terms of dw| [D]."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    D = x.shape[-1]
    c, s = _angles(rope, pos, D)
    d = np.swapaxes(np.asarray(d, dtype=np.float64), -3, -2)
    d1, d2 = d[..., :D // 2], d[..., D // 2:]
    g = np.concatenate([d1 * c + d2 * s, d2 * c - d1 * s], axis=-1)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    terms = (g * n).reshape(-1, D)
    h = g * w
    return r * (h - n * (h * n).mean(-1, keepdims=True)), terms.sum(0), np.abs(terms).sum(0)
