"""Batches over 8-bit cache pages for the GPU tests, with their float64 reference."""

from __future__ import annotations

import numpy as np
import torch

import batch_harness as bh
from oracle import batch as ob
from oracle import cache8 as oc
from paper_2608_00814_amd import ooo


def make_pool(x: np.ndarray):
    """Codes and scales of values [..., R, D], block by block."""
    blocks = x.reshape(*x.shape[:-2], x.shape[-2] // oc.BLOCK, oc.BLOCK, x.shape[-1])
    amax = np.abs(blocks).max(axis=(-1, -2))
    e = np.clip(np.ceil(np.log2(np.maximum(amax, 1e-300) / 448.0)), oc.LEAST, oc.MOST).astype(int)
    codes = oc.round8(blocks * np.exp2(-e.astype(np.float64))[..., None, None]).reshape(x.shape)
    return codes, (e + 127).astype(np.uint8)


class Batch8(bh.Batch):
    """A batch with ragged rows and lengths over 8-bit pages (gap, scale_gap: bytes between pages; quick: any
    numbers, made on the device)."""

    def __init__(self, dt, Hq, Hkv, D, page, rows, lens, layers=0, scale_gap=0, gap=0, seed=0, spread=0.6,
                 quick=False, **kw):
        super().__init__(dt, Hq, Hkv, D, page, rows, lens, seed=seed, **kw)
        r = np.random.default_rng(seed + 1)
        lead = (layers,) if layers else ()
        P, B = self.k.shape[0], page // oc.BLOCK
        shape = (*lead, P, Hkv, page, D)
        n = Hkv * page * D
        self.pools = []
        for _ in range(2):
            if quick:
                c = torch.randint(0, 0x40, shape, dtype=torch.uint8, device="cuda")
                c += torch.randint(0, 2, shape, dtype=torch.uint8, device="cuda") * 128
                s = torch.randint(126, 129, (*lead, P, Hkv, B), dtype=torch.uint8, device="cuda")
                self.pools.append((c, s))
                continue
            x = r.standard_normal(shape) * np.exp(spread * r.standard_normal((*shape[:-1], 1)))
            codes, scales = make_pool(x)
            c = torch.full((*lead, P, n + gap), 0x7F, dtype=torch.uint8, device="cuda")
            c[..., :n] = torch.from_numpy(codes).cuda().reshape(*lead, P, n)
            s = torch.full((*lead, P, Hkv * B + scale_gap), 0xFF, dtype=torch.uint8, device="cuda")
            s[..., :Hkv * B] = torch.from_numpy(scales).cuda().reshape(*lead, P, Hkv * B)
            self.pools.append((c[..., :n].unflatten(-1, (Hkv, page, D)), s[..., :Hkv * B].unflatten(-1, (Hkv, B))))
        (self.k, self.ks), (self.v, self.vs) = self.pools
        self.bind()

    def bind(self):
        pages = (self.k[0] if self.k.dim() == 5 else self.k).view(torch.float8_e4m3fn)
        self.batch = ooo.PagedBatch(self.d_row_start, self.d_len, self.d_table, pages, self.Hq, self.n_rows,
                                    shared_pages=self.d_shared, shared_len=self.shared, anc_mask=self.d_mask,
                                    dtype=self.dt)
        f8 = torch.float8_e4m3fn
        self.cache = ooo.Cache8(self.batch, self.k.view(f8), self.v.view(f8), self.ks, self.vs)

    def bytes(self, layer=None):
        """The pools as NumPy: [(codes, scales) of K, of V]."""
        at = slice(None) if layer is None else layer
        return [(c[at].cpu().numpy().copy(), s[at].cpu().numpy().copy()) for c, s in
                ((self.k, self.ks), (self.v, self.vs))]

    def attend(self, out=None, ws=None, stream=None, layer=0):
        out = torch.full_like(self.q, 7.0) if out is None else out
        plan = ooo.paged_plan8(self.batch, stream=stream)
        if ws is None:
            ws = torch.full((ooo.paged_attn8_workspace(self.batch),), 0xFF, dtype=torch.uint8, device="cuda")
        ooo.paged_attn8(self.batch, self.cache, plan, self.q, self.scale, out, ws, layer=layer, stream=stream)
        return out

    def reference(self, layer=None):
        k, v = (oc.values(*p) for p in self.bytes(0 if layer is None and self.k.dim() == 5 else layer))
        q = self.q.double().cpu().numpy()[:self.total]
        return ob.attention(q, k, v, self.row_start, self.lens, self.table, self.shared_ids, self.shared, self.mask,
                            self.scale)
