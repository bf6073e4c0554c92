"""Batches over cache pages for the GPU tests, with their float64 reference."""

from __future__ import annotations

import math
import random

import numpy as np
import torch

from oracle import batch as ob
from paper_2608_00814_amd import ooo

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -24  # half a step of float32, relative
HALF = {"bf16": 2.0 ** -8, "f32": U32}  # half a step of the stored type


def parents(r: random.Random, n: int):
    return [-1] + [i - 1 if r.random() < 0.7 else r.randrange(i) for i in range(1, n)]


def trie_masks(r: random.Random, rows, words):
    out, depth = [], []
    for n in rows:
        p, d = parents(r, n) if n else [], []
        m = np.zeros((n, words), np.uint64)
        for i in range(n):
            if p[i] >= 0:
                m[i] = m[p[i]]
            m[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
            d.append(0 if p[i] < 0 else d[p[i]] + 1)
        out.append(m)
        depth += d
    return np.concatenate(out), np.array(depth, np.int32)


class Batch:
    """A batch with ragged rows and lengths over randomly placed pages."""

    def __init__(self, dt, Hq, Hkv, D, page, rows, lens, shared=0, mask=None, pad=0, seed=0, spare=1, gap=0,
                 table_pad=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = np.random.default_rng(seed)
        self.dt, self.Hq, self.Hkv, self.D, self.page = TYPES[dt], Hq, Hkv, D, page
        self.kind, self.rows, self.lens, self.shared = dt, list(rows), list(lens), shared
        self.total = sum(rows)
        self.n_rows = max(self.total + pad, 1)
        need = [(n + m + page - 1) // page for n, m in zip(rows, lens)]
        ns = (shared + page - 1) // page
        n_pages = sum(need) + ns + spare
        ids = r.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(rows), max(max(need), 1) + table_pad), -7, np.int32)  # unused entries are no pages
        at = ns
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.shared_ids = ids[:ns]
        self.row_start = np.cumsum([0] + list(rows)).astype(np.int32)
        self.mask = mask  # uint64 [total][words] or None
        shape = (n_pages, Hkv, page, D)
        def pool():
            flat = torch.randn((n_pages, Hkv * page * D + gap), generator=g, device="cuda").to(self.dt)
            return flat[:, :Hkv * page * D].view(shape) if gap == 0 else flat.as_strided(
                shape, (Hkv * page * D + gap, page * D, D, 1))
        self.k, self.v = pool(), pool()
        self.q = torch.randn((self.n_rows, Hq, D), generator=g, device="cuda").to(self.dt)
        self.scale = 1.0 / math.sqrt(D)
        self.d_row_start = torch.from_numpy(self.row_start).cuda()
        self.d_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.d_table = torch.from_numpy(self.table).cuda()
        self.d_shared = torch.from_numpy(self.shared_ids).cuda() if ns else None
        self.d_mask = None
        if mask is not None:
            full = np.zeros((self.n_rows, mask.shape[1]), np.uint64)
            full[:self.total] = mask
            self.d_mask = torch.from_numpy(full.view(np.int64)).cuda()
        self.batch = ooo.PagedBatch(self.d_row_start, self.d_len, self.d_table, self.k, Hq, self.n_rows,
                                    shared_pages=self.d_shared, shared_len=shared, anc_mask=self.d_mask)

    def attend(self, out=None, ws=None, stream=None):
        out = torch.full_like(self.q, 7.0) if out is None else out
        plan = ooo.paged_plan(self.batch, stream=stream)
        if ws is None:
            ws = torch.full((ooo.paged_attn_workspace(self.batch),), 0xFF, dtype=torch.uint8, device="cuda")
        ooo.paged_attn(self.batch, plan, self.q, self.k, self.v, self.scale, out, ws, stream=stream)
        return out

    def reference(self):
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        return ob.attention(f(self.q)[:self.total], f(self.k), f(self.v), self.row_start, self.lens, self.table,
                            self.shared_ids, self.shared, self.mask, self.scale)

    def bound(self, ref, A, S):
        """Largest error of an output: its own rounding, the rounding of the
        probabilities (bf16: half a step each, so of the output at most that
        share of sum p |v|), and float32 sums: scores of D products (relative
        to p twice their error, with l), n keys."""
        n = self.shared + max((a + b for a, b in zip(self.rows, self.lens)), default=0)
        f32 = 2 * (self.D + 8) * U32 * S[..., None] + (n + 64) * U32
        p = HALF["bf16"] if self.kind == "bf16" else 0.0
        h = HALF[self.kind]
        return h * np.abs(ref) + (1 + h) * A * (p + f32) * (1 + 2 * p) + 1e-30

    def check(self, out):
        got = out.double().cpu().numpy()
        if self.total < self.n_rows:
            assert (got[self.total:] == 7.0).all(), "rows behind the last sequence were written"
        ref, A, S = self.reference()
        err = np.abs(got[:self.total] - ref)
        lim = self.bound(ref, A, S)
        assert np.isfinite(got[:self.total]).all()
        assert (err <= lim).all(), (float((err / lim).max()), np.argwhere(err > lim)[:4])


def ragged(r: random.Random, n, most, zero=True):
    v = [r.randint(0 if zero else 1, most) for _ in range(n)]
    if most > 0 and sum(v) == 0:
        v[-1] = most
    return v
