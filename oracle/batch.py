"""Float64 reference of the batched step: append, attention, compaction and
sampling, one row at a time from their definitions (no shared code with the
library).  A pool of pages is ``[n_pages][Hkv][page_rows][D]``; ``place`` is
the only statement of where a token lives."""

from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np


def place(table_row: Sequence[int], token: int, page_rows: int) -> Tuple[int, int]:
    return int(table_row[token // page_rows]), token % page_rows


def append_row(x: np.ndarray, pos: int, Hq: int, Hkv: int, D: int, q_norm, k_norm, eps: float, theta: float):
    """One row [(Hq + 2 Hkv) D] -> q [Hq][D], k [Hkv][D], v [Hkv][D] and the
    sizes |a| + |b| of the rotated pairs (for error bounds of q and k)."""
    h = np.asarray(x, np.float64).reshape(Hq + 2 * Hkv, D).copy()
    for heads, w in ((slice(0, Hq), q_norm), (slice(Hq, Hq + Hkv), k_norm)):
        if w is not None:
            t = h[heads]
            h[heads] = t / np.sqrt((t * t).mean(axis=1, keepdims=True) + eps) * np.asarray(w, np.float64)
    ang = pos * theta ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(ang), np.sin(ang)
    t = h[:Hq + Hkv]
    a, b = t[:, :D // 2], t[:, D // 2:]
    turned = np.concatenate([a * c - b * s, b * c + a * s], axis=1)
    size = np.concatenate([np.abs(a) + np.abs(b)] * 2, axis=1)
    return turned[:Hq], turned[Hq:], h[Hq + Hkv:], size[:Hq], size[Hq:]


def attention_row(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """q [D], the keys k [n][D] it sees and their v: (output, sum of p |v|,
    largest |score| term sum) - zeros where n is 0."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros(q.shape[0]), np.zeros(q.shape[0]), 0.0
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ v, p @ np.abs(v), float((abs(scale) * (np.abs(k) @ np.abs(q))).max())


def visible(i: int, rows: int, mask_row: Optional[Sequence[int]]) -> List[int]:
    """New rows that row i of a sequence sees."""
    if mask_row is None:
        return list(range(i + 1))
    return [j for j in range(min(rows, 64 * len(mask_row))) if (int(mask_row[j // 64]) >> (j % 64)) & 1]


def attention(q, k_pool, v_pool, row_start, seq_len, table, shared_pages, shared_len, mask, scale):
    """q [rows][Hq][D] of all sequences -> (out, bound terms A [rows][Hq][D]
    and S [rows][Hq])."""
    rows, Hq, D = q.shape
    Hkv, R = k_pool.shape[1], k_pool.shape[2]
    G = Hq // Hkv
    out, A, S = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    sp = [place(shared_pages, t, R) for t in range(shared_len)]
    for b in range(len(seq_len)):
        n = row_start[b + 1] - row_start[b]
        own = [place(table[b], t, R) for t in range(seq_len[b] + n)]
        for i in range(n):
            r = row_start[b] + i
            at = sp + own[:seq_len[b]] + [own[seq_len[b] + j]
                                          for j in visible(i, n, None if mask is None else mask[r])]
            pg, sl = [a[0] for a in at], [a[1] for a in at]
            for g in range(Hkv):
                kk, vv = k_pool[pg, g, sl], v_pool[pg, g, sl]
                for h in range(g * G, (g + 1) * G):
                    out[r, h], A[r, h], S[r, h] = attention_row(q[r, h], kk, vv, scale)
    return out, A, S


def compact(pool: np.ndarray, row_start, seq_len, table, path, accept) -> np.ndarray:
    """One layer's pool [n_pages][Hkv][R][D] after the accepted rows moved."""
    old, new, R = pool, pool.copy(), pool.shape[2]
    for b in range(len(seq_len)):
        if accept[b] < 0 or accept[b] >= path.shape[1]:
            continue
        for d in range(accept[b] + 1):
            src, dst = place(table[b], seq_len[b] + path[b, d], R), place(table[b], seq_len[b] + d, R)
            new[dst[0], :, dst[1]] = old[src[0], :, src[1]]
    return new


def sample(x: np.ndarray, T: float, k: int, top_p: float, min_p: float, u: float):
    """(id, probability, kept) for one row of logits."""
    x = np.asarray(x, np.float64)
    live = [i for i in range(len(x)) if x[i] == x[i] and x[i] != -math.inf]
    if not live:
        return -1, 0.0, 0
    live.sort(key=lambda i: (-x[i], i))
    top = x[live[0]]
    greedy = not T > 0
    w = [1.0 if x[i] == top else math.exp((x[i] - top) / (1.0 if greedy else T)) for i in live]
    n = 1 if greedy else min(k, len(live)) if k > 0 else len(live)
    if top_p < 1:
        want = max(top_p, 0.0) * math.fsum(w[:n])
        run, n_p = 0.0, 0
        for n_p, cum in enumerate(np.cumsum(w[:n]), 1):
            if cum >= want:
                break
        n = min(n, n_p)
    if min_p > 0:
        n = min(n, max(1, sum(1 for a in w if a >= min_p)))
    cum = np.cumsum(w[:n])
    at = min(n - 1, int(np.searchsorted(cum, max(u, 0.0) * cum[-1], side="right")))
    return live[at], w[at] / cum[-1], n
