"""Float64 reference of the 8-bit cache: numbers and scales from their
definitions, append, compaction and fork row by row (no shared code with the
library).  A pool is a pair of bytes: codes [n_pages][Hkv][page_rows][D] and
scales [n_pages][Hkv][page_rows / 32]."""

from __future__ import annotations

import math
from fractions import Fraction
from typing import Tuple

import numpy as np

from oracle.batch import place

BLOCK, LEAST, MOST = 32, -100, 119


def _number(code: int) -> float:
    """The e4m3 number of a byte: sign, 4 bits of exponent (bias 7), 3 of fraction; all ones is NaN."""
    e, f = code >> 3 & 15, code & 7
    if e == 15 and f == 7:
        return float("nan")
    x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
    return -x if code & 128 else x


NUMBERS = np.array([_number(c) for c in range(256)])
_POS = NUMBERS[:127]  # 0 .. 448, rising with the code


def round8(x: np.ndarray) -> np.ndarray:
    """Codes of the numbers nearest to x (ties: even code), bounded to 448; NaN where x is not finite."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    hi = np.searchsorted(_POS, a, side="left")
    lo = np.maximum(hi - 1, 0)
    up = _POS[hi] - a, a - _POS[lo]  # exact: the numbers are multiples of 2^-9
    code = np.where(up[0] < up[1], hi, np.where(up[1] < up[0], lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(a == _POS[hi], hi, code)
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def exponent(amax: float) -> int:
    """The least e in LEAST .. MOST with amax <= 448 2^e (MOST where none is)."""
    e = LEAST if amax <= 0 else min(max(math.frexp(amax)[1] - 12, LEAST), MOST)  # amax > 448 2^(e - 1)
    while e < MOST and Fraction(amax) > 448 * Fraction(2) ** e:
        e += 1
    return e


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What a pool's numbers stand for."""
    up = np.exp2(scales.astype(np.float64) - 127)
    return NUMBERS[codes] * np.repeat(up, BLOCK, axis=-1)[..., None]


def finite_max(x: np.ndarray) -> float:
    a = np.abs(x)
    return float(np.max(np.where(np.isfinite(a), a, 0.0), initial=0.0))


def append(codes, scales, rows, table, seq_len, page_rows, exps=None) -> Tuple[np.ndarray, np.ndarray]:
    """One sequence's new rows [n][Hkv][D] (float64) into a pool, in place.
    ``exps``: scale exponents to take in place of the computed ones, by (page,
    head, block), where float32 sizes may have fallen on the other side of a
    bound."""
    n, Hkv, _ = rows.shape
    t = 0
    while t < n:
        token = seq_len + t
        m = min(n - t, BLOCK - token % BLOCK)
        page, sl = place(table, token, page_rows)
        blk, lo, held = sl // BLOCK, sl // BLOCK * BLOCK, (sl % BLOCK if t == 0 else 0)
        for g in range(Hkv):
            e = exponent(finite_max(rows[t:t + m, g])) if exps is None else exps[page, g, blk]
            if held:
                was = int(scales[page, g, blk]) - 127
                e = max(e, was)
                if e != was:
                    codes[page, g, lo:sl] = round8(NUMBERS[codes[page, g, lo:sl]] * 2.0 ** (was - e))
            with np.errstate(over="ignore", invalid="ignore"):
                codes[page, g, sl:sl + m] = round8(rows[t:t + m, g] * 2.0 ** -e)
            scales[page, g, blk] = e + 127
        t += m
    return codes, scales


def compact(codes, scales, row_start, seq_len, table, path, accept, page_rows):
    """One layer's pool after the accepted rows moved."""
    oc, os_ = codes, scales
    codes, scales = codes.copy(), scales.copy()
    for b in range(len(seq_len)):
        n = row_start[b + 1] - row_start[b]
        if accept[b] < 0 or accept[b] >= path.shape[1]:
            continue
        blocks = {}
        for d in range(min(int(accept[b]) + 1, n)):
            i = int(path[b, d])
            if 0 <= i < n:
                blocks.setdefault((seq_len[b] + d) // BLOCK, []).append((seq_len[b] + d, seq_len[b] + i))
        for blk, moves in blocks.items():
            first = blk * BLOCK
            moves += [(t, t) for t in range(first, min(seq_len[b], first + BLOCK))]
            at = [(place(table[b], to, page_rows), place(table[b], fr, page_rows)) for to, fr in moves]
            for g in range(codes.shape[1]):
                exps = [int(os_[fp, g, fs // BLOCK]) - 127 for _, (fp, fs) in at]
                for ((tp, ts), (fp, fs)), e in zip(at, exps):
                    codes[tp, g, ts] = round8(NUMBERS[oc[fp, g, fs]] * 2.0 ** (e - max(exps)))
                scales[at[0][0][0], g, at[0][0][1] // BLOCK] = max(exps) + 127
    return codes, scales


def fork(seq_len, table, parent, fresh, n_pages, page_rows, in_place):
    """New lengths and tables, and the copies (child, from page, to page, rows)."""
    n, ld = table.shape
    lens, out, copies = list(seq_len), table.copy(), []
    for b in range(n):
        p = int(parent[b])
        if p < 0 or p == b or p >= n or not 0 <= fresh[b] < n_pages or not 0 <= seq_len[p] < ld * page_rows:
            continue
        if in_place and 0 <= parent[p] < n and parent[p] != p:
            continue
        full, rows = divmod(int(seq_len[p]), page_rows)
        if rows:
            if not 0 <= table[p, full] < n_pages:
                continue
            copies.append((b, int(table[p, full]), int(fresh[b]), rows))
        lens[b] = int(seq_len[p])
        out[b, :full] = table[p, :full]
        out[b, full] = fresh[b]
    return np.array(lens, np.int32), out, copies
