"""The 8-bit cache's append past the rows up to which a block's heads are shared out among workgroups
(csrc/cache8.hip, kFewRows), compactions over several windows of 256 rows, commits against direct appends, and
forks of parents without parents."""

import random

import numpy as np
import pytest
import torch

from oracle import batch as ob
from oracle import cache8 as oc
from paper_2608_00814_amd import ooo

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import batch_harness as bh
    from batch_harness import TYPES, ragged
    from cache8_harness import Batch8
    from test_gpu_cache8 import Forks, check_compact, run_append

FEW = 4096


def sized(n, width, dt, seed):
    """Rows of sizes from far below to far above what the pool's scales are for."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, width), generator=g, device="cuda")
    by = torch.tensor([0.01, 1.0, 30.0, 600.0, 5000.0], device="cuda")
    return (x * by[torch.randint(0, 5, (n, 1), generator=g, device="cuda")]).to(TYPES[dt])


def to_sum(r, n, most, total):
    """n counts of up to `most`, none and ones among them, that sum to `total`."""
    rows = [r.choice([0, 1, r.randint(2, most)]) for _ in range(n)]
    at = 0
    while sum(rows) != total:
        gap = total - sum(rows)
        rows[at % n] = min(max(rows[at % n] + gap, 0), most)
        at += 1
    return rows


@pytest.mark.parametrize("total", [FEW, FEW + 1, FEW + 700])
@pytest.mark.parametrize("dt,Hq,Hkv,D,norm", [("bf16", 5, 5, 64, True), ("bf16", 10, 5, 128, False),
                                             ("f32", 6, 6, 64, False), ("f32", 7, 7, 128, True)])
def test_append_of_long_batches(dt, Hq, Hkv, D, norm, total):
    """Five to seven heads: a wave of the one workgroup has K and V of several, one behind the other."""
    r = random.Random(total)
    rows = to_sum(r, 40, 300, total)
    lens = ragged(r, 40, 150)
    lens[:4] = [0, 31, 32, 63]
    b = Batch8(dt, Hq, Hkv, D, 64, rows, lens, shared=9, pad=3, scale_gap=1, quick=True)
    assert run_append(b, norm, None, qkv=sized(b.n_rows, (Hq + 2 * Hkv) * D, dt, 3)) > 0


@pytest.mark.parametrize("dt,Hkv,D", [("bf16", 20, 128), ("bf16", 33, 64), ("f32", 9, 128)])
def test_append_of_one_row_of_very_many_sequences(dt, Hkv, D):
    """Three groups of heads: a wave has two of the six tasks of K and V."""
    n = FEW + 4
    b = Batch8(dt, Hkv, Hkv, D, 32, [1] * n, [(7 * i) % 50 for i in range(n)], pad=2, quick=True)
    assert run_append(b, True, None, qkv=sized(b.n_rows, 3 * Hkv * D, dt, 4)) > 0


def long_paths(r, rows, kind):
    """One root path a sequence, strictly rising, of 300 rows or more where the sequence has them."""
    cap = max(rows) + 1
    path, acc = np.full((len(rows), cap), -1, np.int32), np.zeros(len(rows), np.int32)
    for s, n in enumerate(rows):
        if kind == "dense":
            p = list(range(n))
        elif kind == "shift":  # every row behind the root comes from 1 to 40 rows on
            p = [0] + list(range(1 + r.randint(1, 40), n))
        elif kind == "late":   # rows stay up to 255 and move from there on
            p = list(range(min(n, 256))) + list(range(min(n, 256) + r.randint(1, 9), n))
        else:
            p = [0] + sorted(r.sample(range(1, n), (3 * n) // 4))
        path[s, :len(p)], acc[s] = p, len(p) - 1
    return path, acc


@pytest.mark.parametrize("kind", ["dense", "shift", "late", "sparse"])
@pytest.mark.parametrize("D,page", [(64, 32), (128, 32), (64, 128), (128, 128)])
def test_compact_over_several_windows(D, page, kind):
    """Windows begin at 256 rows from the first touched block on: lengths at a block's begin and end, and scales
    that differ from block to block on both sides of a window's end."""
    r = random.Random(page + D)
    rows, lens = [700, 420, 300, 513, 257, 225, 2], [0, 31, 32, 95, 64, 31, 40]
    b = Batch8("bf16", 2, 2, D, page, rows, lens, layers=2, gap=32, scale_gap=2, seed=page, spread=2.0)
    check_compact(b, *long_paths(r, rows, kind))


def test_compact_leaves_bad_entries_of_later_windows():
    r = random.Random(1)
    rows, lens = [700, 600], [31, 64]
    b = Batch8("bf16", 2, 2, 64, 32, rows, lens, seed=3, spread=2.0)
    path, acc = long_paths(r, rows, "sparse")
    path[0, 300], path[0, 400], path[1, 257] = 700, -3, 1 << 30  # not rows: they stay where they are
    check_compact(b, path, acc)


def commit(b, qkv, path, acc, depth):
    q = torch.empty((b.n_rows, b.Hq, b.D), dtype=b.dt, device="cuda")
    ooo.paged_append8(b.batch, b.cache, qkv, None, None, 1e-6, 1e6, q, depth=torch.from_numpy(depth).cuda())
    if path is not None:
        ooo.paged_compact8(b.batch, b.cache, torch.from_numpy(path).cuda(), torch.from_numpy(acc).cuda())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_commit_against_a_direct_append(dt):
    """A trie appended and its accepted rows committed, against an append of the accepted rows alone.  Rejected rows
    may leave a larger scale behind (e against e'), never a smaller one.  A number whose size is 2^(e - 6) or more is
    normal under both scales and so rounded alike.  Any other one is rounded to steps of 2^(e - 9) or finer: when it
    is appended, again when it is put under e, and in the direct append: 3 2^(e - 10) at most between the two.  (A
    rotated key may come from another form of the same float32 products: then it may also be the next number.)"""
    r = random.Random(4)
    rows, lens, Hkv, D, R = [50, 40, 64, 9, 1], [30, 0, 64, 95, 33], 2, 64, 32
    mask, depth = bh.trie_masks(r, rows, 1)
    path, acc = np.full((5, 65), -1, np.int32), np.zeros(5, np.int32)
    for s, n in enumerate(rows):
        at = int(np.cumsum([0] + rows)[s])
        node = max(range(n), key=lambda j: depth[at + j])
        p = [j for j in range(n) if (int(mask[at + node, 0]) >> j) & 1]
        path[s, :len(p)], acc[s] = p, len(p) - 1
    starts = np.cumsum([0] + rows)
    a = Batch8(dt, 2, Hkv, D, R, rows, lens, shared=20, seed=2, spread=0.3)
    # sizes from 1 to 1000 for rejected rows, near 1 for the others
    qkv = sized(a.n_rows, 6 * D, dt, 5)
    kept = np.concatenate([starts[s] + path[s, :acc[s] + 1] for s in range(5)])
    x = torch.randn((len(kept), 6 * D), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    qkv[torch.from_numpy(kept).cuda()] = x.to(a.dt)
    few = [int(n) + 1 for n in acc]
    d = Batch8(dt, 2, Hkv, D, R, few, lens, shared=20, seed=2, spread=0.3)
    d.table = a.table.copy()
    d.d_table = torch.from_numpy(d.table).cuda()
    d.k, d.v, d.ks, d.vs = a.k.clone(), a.v.clone(), a.ks.clone(), a.vs.clone()
    d.bind()
    commit(a, qkv, path, acc, depth)
    commit(d, qkv[torch.from_numpy(kept).cuda()].contiguous(), None, None,
           np.concatenate([np.arange(n, dtype=np.int32) for n in few]))
    coarser = differ = 0
    for kv, (ca, sa), (cd, sd) in zip((0, 1), a.bytes(), d.bytes()):
        va, vd = oc.values(ca, sa), oc.values(cd, sd)
        for s, n in enumerate(few):
            for t in range(lens[s] // 32 * 32, lens[s] + n):
                page, row = ob.place(a.table[s], t, R)
                e, e1 = (x[page, :, row // 32].astype(int) - 127 for x in (sa, sd))
                assert (e >= e1).all()
                up, y, z = np.exp2(e.astype(float))[:, None], va[page, :, row], vd[page, :, row]
                normal = np.abs(z) >= up * 2.0 ** -6
                next_ = np.abs(z) / 8 if kv == 0 else 0.0
                assert kv == 0 or np.array_equal(y[normal], z[normal])
                assert (np.abs(y - z) <= 3 * up * 2.0 ** -10 + next_).all()
                coarser += (e > e1).sum()
                differ += (y != z).sum()
    assert coarser > 0 and differ > 0


@pytest.mark.parametrize("kind", ["f8", "bf16"])
def test_fork_in_place_of_a_parent_whose_own_parent_is_none(kind):
    """An entry past the sequences names none: its sequence is left as it is, and its children continue it."""
    f = Forks(kind, [40, 7, 64, 33], 32)
    assert len(f.check([4, 0, 1 << 30, 2], True)) == 1 and f.d_len.tolist() == [40, 40, 64, 64]
