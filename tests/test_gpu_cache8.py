"""The 8-bit cache's entry points, and fork, on the GPU against the float64 reference."""

import math
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
    from batch_harness import HALF, U32, Batch, ragged
    from cache8_harness import Batch8


def f64(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------ append


def run_append(b, norm, depth, seed=1, ld_gap=0, theta=1e6, qkv=None, layer=0, spread=1.0):
    """Appends random rows of sizes that vary and checks q, codes, scales and that nothing else changed."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (b.Hq + 2 * b.Hkv) * b.D
    if qkv is None:
        x = torch.randn((b.n_rows, width), generator=g, device="cuda")
        x = (x * torch.exp(spread * torch.randn((b.n_rows, 1), generator=g, device="cuda"))).to(b.dt)
        qkv = torch.full((b.n_rows, width + ld_gap), float("nan"), dtype=b.dt, device="cuda")[:, :width]
        qkv.copy_(x)
    qw, kw = ((torch.randn(b.D, generator=g, device="cuda") * 0.1 + 1).to(b.dt) if norm else None for _ in range(2))
    d = None if depth is None else torch.from_numpy(depth).cuda()
    q_out = torch.full((b.n_rows, b.Hq, b.D), 7.0, dtype=b.dt, device="cuda")
    before = b.bytes()
    ooo.paged_append8(b.batch, b.cache, qkv, qw, kw, 1e-6, theta, q_out, depth=d, layer=layer)
    after = b.bytes()
    got_q, x = f64(q_out), f64(qkv)
    nq, nk = (None, None) if not norm else (f64(qw), f64(kw))
    assert (got_q[b.total:] == 7.0).all()
    h, grown = HALF[b.kind], 0
    for kv in range(2):
        (c0, s0), (c1, s1) = before[kv], after[kv]
        if c0.ndim == 5:
            for l in range(c0.shape[0]):
                assert l == layer or (np.array_equal(c0[l], c1[l]) and np.array_equal(s0[l], s1[l]))
            c0, s0, c1, s1 = c0[layer], s0[layer], c1[layer], s1[layer]
        for s in range(len(b.rows)):
            n, m = b.rows[s], b.lens[s]
            rows, off = np.zeros((n, b.Hkv, b.D)), np.zeros((n, b.Hkv, b.D))
            for i in range(n):
                r = b.row_start[s] + i
                pos = b.shared + m + (i if depth is None else int(depth[r]))
                with np.errstate(invalid="ignore"):
                    q, k, v, sq, sk = ob.append_row(x[r], pos, b.Hq, b.Hkv, b.D, nq, nk, 1e-6, theta)
                # norm factor, sine and cosine and two products in float32: under 64 roundings of the pair
                rows[i], off[i] = (v, 0.0) if kv else (k, 64 * U32 * sk)
                if kv == 0:
                    fine = np.isfinite(q)
                    # below 2^-126 a step is no share of the value: half of the least one, 2^-134 in bf16, and
                    # in float32 2^-150 for each of the pair's two products, their sum and the stored value
                    tiny = (2.0 ** -134 if b.kind == "bf16" else 0.0) + 4 * 2.0 ** -150
                    assert (np.abs(got_q[r] - q) <= h * np.abs(q) + 64 * U32 * sq + tiny)[fine].all(), (s, i)
                    assert not np.isfinite(got_q[r][~fine]).any()
            exps = {}
            for blk in {(m + i) // 32 for i in range(n)}:
                i0, i1 = max(32 * blk - m, 0), min(32 * blk + 32 - m, n)
                page, sl = ob.place(b.table[s], 32 * blk, b.page)
                for g_ in range(b.Hkv):
                    fine = np.isfinite(rows[i0:i1, g_])
                    a, o = np.abs(rows[i0:i1, g_][fine]), np.broadcast_to(off[i0:i1, g_], fine.shape)[fine]
                    lo, hi = (oc.exponent(max(float(np.max(a - o, initial=0.0)), 0.0)),
                              oc.exponent(float(np.max(a + o, initial=0.0))))
                    held = 32 * blk < m
                    was = int(s0[page, g_, sl // 32]) - 127
                    e = int(s1[page, g_, sl // 32]) - 127
                    assert (max(lo, was) if held else lo) <= e <= (max(hi, was) if held else hi), (s, blk, g_)
                    grown += held and e > was
                    exps[page, g_, sl // 32] = e
            oc.append(c0, s0, rows, b.table[s], m, b.page, exps)
            for i in range(n):  # a new row's numbers: the nearest, but for the float32 error
                page, sl = ob.place(b.table[s], m + i, b.page)
                e = s1[page, :, sl // 32].astype(float)[:, None] - 127
                y, want = oc.NUMBERS[c1[page, :, sl]], rows[i] * 2.0 ** -e
                o = off[i] * 2.0 ** -e
                with np.errstate(invalid="ignore", divide="ignore"):
                    top = np.minimum(np.abs(want) + o, 448.0)
                    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(top, 1e-300))), -6) - 3)
                    fine = np.isfinite(want)
                    ok = (np.abs(y - np.clip(want, -448, 448)) <= step / 2 + o) | (~fine & np.isnan(y))
                assert ok.all(), (kv, s, i, y[~ok], want[~ok])
                if kv == 1:
                    assert np.array_equal(c0[page, :, sl][fine], c1[page, :, sl][fine])  # values go in unchanged
                c0[page, :, sl] = c1[page, :, sl]
        assert np.array_equal(c0, c1), "bytes of other rows changed, or committed rows were put wrongly"
        assert np.array_equal(s0, s1), "a scale of another block changed"
    return grown


@pytest.mark.parametrize("dt,Hq,Hkv,D,page,norm,trie", [
    ("bf16", 32, 8, 128, 64, True, False), ("bf16", 40, 8, 128, 32, True, True), ("bf16", 14, 2, 64, 32, False, False),
    ("bf16", 3, 1, 128, 128, True, False), ("bf16", 40, 20, 64, 32, False, False), ("f32", 4, 1, 64, 32, True, True),
    ("f32", 16, 8, 128, 32, False, False), ("f32", 5, 5, 128, 64, True, False), ("f32", 18, 9, 64, 32, False, False),
])
def test_append(dt, Hq, Hkv, D, page, norm, trie):
    r = random.Random(3)
    rows = ragged(r, 9, 70)
    rows[0] = rows[4] = 0
    rows[1:3] = [1, 33]
    lens = ragged(r, 9, 150)
    lens[3], lens[5] = 32, 95
    depth = None
    if trie:
        depth = np.concatenate([bh.trie_masks(r, rows, 2)[1], np.full(3, 99, np.int32)])
    run_append(Batch8(dt, Hq, Hkv, D, page, rows, lens, shared=77, pad=3, gap=64, scale_gap=3), norm, depth, ld_gap=16)


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("rows", [1, 2, 31])
def test_append_scales_grow_under_committed_rows(dt, D, rows):
    """Rows 1/100 to 10^5 times the committed ones: codes stay, become subnormal, become zero."""
    lens = [1, 5, 31, 32, 33, 63, 40, 20]
    b = Batch8(dt, 6, 3, D, 32, [rows] * 8, lens, seed=rows)
    qkv = torch.randn((8, rows, 12 * D), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    qkv *= torch.tensor([0.01, 10, 3000, 1, 100, 400, 1e5, 30], device="cuda")[:, None, None]
    assert run_append(b, False, None, qkv=qkv.view(8 * rows, 12 * D).to(b.dt)) >= 6 * 3 * 2


def test_append_one_row_of_many_sequences():
    r = random.Random(5)
    b = Batch8("bf16", 2, 1, 64, 32, [1] * 300, ragged(r, 300, 70), shared=5)
    run_append(b, False, None)
    b = Batch8("f32", 2, 1, 64, 32, ragged(r, 300, 2), ragged(r, 300, 40), shared=5)
    run_append(b, True, None)


def test_append_many_rows():
    """More than 2048 rows: a workgroup goes over several of them."""
    r = random.Random(6)
    rows = ragged(r, 30, 160)
    rows[3] = 0
    assert sum(rows) > 2048
    run_append(Batch8("bf16", 2, 1, 64, 64, rows, ragged(r, 30, 90), pad=5), True, None)
    run_append(Batch8("bf16", 1, 1, 64, 32, [1] * 2100, [(7 * i) % 50 for i in range(2100)]), False, None)


def test_append_far_position_and_layers():
    run_append(Batch8("f32", 2, 1, 64, 32, [1], [0], shared=900000), True, None)
    run_append(Batch8("bf16", 4, 2, 64, 32, [3, 40], [3, 31], layers=3, gap=16, scale_gap=1), True, None, layer=1)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_append_odd_values(dt):
    """NaN, infinities, zeros, the smallest and largest values; each in a block of its own, with others."""
    b = Batch8(dt, 1, 1, 64, 32, [1, 1, 2, 40, 3, 1, 2], [0, 5, 30, 0, 64, 40, 33])
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((b.n_rows, 3 * 64), generator=g, device="cuda").to(b.dt)
    qkv[0] = 0                                     # a zero block
    qkv[1, 130] = float("nan")
    qkv[2, 66], qkv[2, 191] = float("inf"), -float("inf")
    qkv[4:44] *= 1e-36                             # below the least scale
    qkv[44:47] *= 1e37                             # 3e37 or so: scales near the largest
    qkv[47, 128:] = torch.finfo(b.dt).max          # beyond 448 2^119
    qkv[48] = float("nan")
    run_append(b, False, None, qkv=qkv, theta=1e30)


def test_append_drops_rows_without_a_page():
    b = Batch8("bf16", 8, 2, 64, 32, [20, 40, 4, 1], [0, 14, 5, 3])
    b.table[1, 1] = b.k.shape[0]  # one past the pool
    b.table[2, 0] = -1
    b.d_table.copy_(torch.from_numpy(b.table))
    b.d_len[0] = 2 ** 30          # past its table
    b.d_len[3] = -4
    width = 12 * 64
    qkv = torch.randn((b.n_rows, width), device="cuda").to(b.dt)
    q_out = torch.full((b.n_rows, 8, 64), 7.0, dtype=b.dt, device="cuda")
    before = b.bytes()
    ooo.paged_append8(b.batch, b.cache, qkv, None, None, 1e-6, 1e6, q_out)
    good = int(b.table[1, 0])     # 18 rows of sequence 1 lie on its good page
    for (c0, s0), (c1, s1) in zip(before, b.bytes()):
        assert {int(p) for p in np.argwhere((c0 != c1).any(axis=(1, 2, 3)))[:, 0]} == {good}
        assert {int(p) for p in np.argwhere(s0 != s1)[:, 0]} <= {good}
    assert not (f64(q_out) == 7.0).all(axis=2).any()


@pytest.mark.parametrize("starts", [[5, 9, 14], [0, 9, 4], [9, -3, 14], [-4, 9, 1 << 30]])
def test_append_bounds_row_starts(starts):
    b = Batch8("bf16", 2, 1, 64, 32, [9, 5], [0, 0])
    b.d_row_start.copy_(torch.tensor(starts, dtype=torch.int32))
    qkv = torch.randn((b.n_rows, 4 * 64), device="cuda").to(b.dt)
    q_out = torch.full((b.n_rows, 2, 64), 7.0, dtype=b.dt, device="cuda")
    before = b.bytes()
    ooo.paged_append8(b.batch, b.cache, qkv, None, None, 1e-6, 1e6, q_out)
    R = min(max(starts[2], 0), b.n_rows)
    lo = [min(max(s, 0), R) for s in starts]
    places = set()
    for s in range(2):
        places |= {ob.place(b.table[s], i, 32) for i in range(min(max(starts[s + 1], lo[s]), R) - lo[s])}
    for (c0, _), (c1, _) in zip(before, b.bytes()):
        got = {(int(p), int(t)) for p, t in np.argwhere((c0 != c1).any(axis=(1, 3)))}
        assert got <= places
        if starts[0] == 5:  # two sequences of 4 and 5 rows behind 5 that are none's
            assert got == places and (f64(q_out)[:5] == 7.0).all()
    assert (f64(q_out)[R:] == 7.0).all()


# --------------------------------------------------------------- attention


@pytest.mark.parametrize("shared", [0, 1, 63, 64, 200])
@pytest.mark.parametrize("dt,Hq,Hkv,D,page", [
    ("bf16", 8, 2, 128, 32), ("bf16", 14, 2, 64, 64), ("bf16", 5, 1, 128, 128), ("f32", 4, 1, 64, 32),
    ("f32", 6, 2, 128, 128),
])
def test_attn_decode(dt, Hq, Hkv, D, page, shared):
    r = random.Random(shared)
    lens = [0, 1, 15, 31, 32, 63, 64, 65] + ragged(r, 4, 200)
    b = Batch8(dt, Hq, Hkv, D, page, [1] * len(lens), lens, shared=shared, pad=2, seed=shared, scale_gap=shared % 3)
    b.check(b.attend())


@pytest.mark.parametrize("trie", [False, True])
@pytest.mark.parametrize("dt,Hq,Hkv,D,shared,most", [
    ("bf16", 8, 2, 128, 130, 9), ("bf16", 8, 2, 128, 0, 70), ("bf16", 16, 2, 64, 70, 40), ("bf16", 5, 1, 64, 0, 30),
    ("bf16", 40, 1, 128, 33, 8), ("f32", 4, 1, 64, 50, 40), ("f32", 4, 2, 128, 0, 70),
])
def test_attn_ragged_rows(dt, Hq, Hkv, D, shared, most, trie):
    r = random.Random(most)
    rows = ragged(r, 6, most)
    rows[2] = 0
    lens = ragged(r, 6, 140)
    mask = bh.trie_masks(r, rows, (most + 63) // 64)[0] if trie else None
    b = Batch8(dt, Hq, Hkv, D, 32, rows, lens, shared=shared, mask=mask, pad=3, seed=most, gap=32, scale_gap=1)
    b.check(b.attend())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [0, 65])
def test_attn_masks_of_any_shape(dt, shared):
    """Random bits (later rows too), rows that see nothing new, and with no
    prompt and no own tokens rows that see nothing at all: zero."""
    r = np.random.default_rng(7)
    rows, lens = [33, 1, 17, 70], [0, 0, 64, 5]
    mask = r.integers(0, 1 << 63, size=(sum(rows), 2), dtype=np.uint64)
    mask[3] = mask[33] = mask[40] = 0
    b = Batch8(dt, 4, 2, 64, 32, rows, lens, shared=shared, mask=mask, seed=9)
    out = b.attend()
    b.check(out)
    if shared == 0:
        assert not out[3].any() and not out[33].any()


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attn_long_splits(dt, D):
    """Long own caches and a long prompt: many parts to join."""
    for rows, lens, shared in (([1], [3000], 0), ([1, 2], [1500, 10], 2100), ([40, 1], [700, 2000], 900)):
        b = Batch8(dt, 8, 2, D, 64, rows, lens, shared=shared, seed=lens[0])
        b.check(b.attend())


def test_attn_wide_prompt_chunk():
    b = Batch8("bf16", 4, 1, 128, 32, [150, 300], [33, 0], shared=40)
    b.check(b.attend())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("shared", [0, 2601, 9000])
def test_attn_many_pages(dt, D, shared):
    """Hundreds of the smallest pages to a part, in both kinds of it."""
    for rows, lens in (([1, 2], [5003, 3]), ([70, 1], [2100, 4100])):
        b = Batch8(dt, 2, 1, D, 32, rows, lens, shared=shared, seed=shared)
        b.check(b.attend())


@pytest.mark.parametrize("D,rows,lens", [(64, 1, [20000, 3000]), (128, 1, [17000, 500]), (64, 40, [9000, 2500]),
                                         (128, 40, [9000, 60])])
def test_attn_one_worker_goes_over_many_steps(D, rows, lens):
    """As many heads as workgroups: one wave, or one workgroup, has hundreds of
    half-tiles or tiles of one sequence."""
    b = Batch8("bf16", 256, 256, D, 64, [rows, 1], lens, shared=0, seed=D, quick=True)
    got = f64(b.attend())
    heads = [0, 100, 255]
    k, v = (oc.values(c[:, heads].cpu().numpy(), s[:, heads].cpu().numpy()) for c, s in b.pools)
    ref, A, S = ob.attention(f64(b.q)[:, heads], k, v, b.row_start, b.lens, b.table, b.shared_ids, 0, None, b.scale)
    err, lim = np.abs(got[:, heads] - ref), b.bound(ref, A, S)
    assert np.isfinite(got).all() and (err <= lim).all(), float((err / lim).max())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("shared,page", [(0, 32), (333, 32), (1000, 128)])
def test_attn_tries_over_long_sequences(dt, D, shared, page):
    r = random.Random(D)
    rows, lens = [64, 3, 150, 40, 33], [300, 700, 261, 1000, 321]
    mask = bh.trie_masks(r, rows, 3)[0]
    b = Batch8(dt, 8, 2, D, page, rows, lens, shared=shared, mask=mask, pad=1, seed=shared)
    b.check(b.attend())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("long_", [0, 600])
def test_attn_what_is_not_seen_does_not_matter(dt, D, long_):
    """NaN in unused rows and in new rows that a row does not see, and scales of
    blocks that hold no token, leave it as it is; rows that see NaN are not
    finite."""
    r = random.Random(1)
    rows, lens = [12, 40, 1], [10, 77 + long_, 64]
    mask = bh.trie_masks(r, rows, 1)[0]
    b = Batch8(dt, 8, 2, D, 64, rows, lens, shared=30 + long_, mask=mask, seed=4)
    R = b.page
    ends = [(b.table[s], n + m) for s, (n, m) in enumerate(zip(rows, lens))] + [(b.shared_ids, b.shared)]
    for ids, end in ends:  # behind each sequence's and the prompt's end
        for t in range(end, (end + R - 1) // R * R):
            pg, sl = ob.place(ids, t, R)
            b.k[pg, :, sl] = b.v[pg, :, sl] = 0x7F
        for blk in range((end + 31) // 32, (end + R - 1) // R * R // 32):
            pg, sl = ob.place(ids, 32 * blk, R)
            b.ks[pg, :, sl // 32], b.vs[pg, :, sl // 32] = 255, 0
    b.check(b.attend())
    for j in (5, 30, 39):
        pg, sl = ob.place(b.table[1], lens[1] + j, R)
        b.v[pg, :, sl] = 0xFF
        if j == 30:
            b.k[pg, :, sl] = 0x7F
    out = b.attend()
    with np.errstate(invalid="ignore"):
        ref, A, S = b.reference()
    sees = np.array([[(int(mask[x, 0]) >> j) & 1 for j in (5, 30, 39)] for x in range(12, 52)]).any(axis=1)
    assert sees.any() and not sees.all()
    hit = np.zeros(b.total, bool)
    hit[12:52] = sees
    got = f64(out)
    assert not np.isfinite(got[hit]).any(), "a seen value that is not finite was lost"
    with np.errstate(invalid="ignore"):
        err, lim = np.abs(got[~hit] - ref[~hit]), b.bound(ref, A, S)[~hit]
    assert (err <= lim).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 20])
def test_attn_bad_queries_stay_their_own(dt, rows):
    b = Batch8(dt, 8, 2, 64, 32, [rows] * 3, [40, 90, 7], shared=70)
    good = f64(b.attend())
    b.q[rows, 3, 5] = float("nan")
    b.q[rows, 6, 7] = float("inf")
    got = f64(b.attend())
    assert np.isnan(got[rows, [3, 6]]).all()
    ref, A, S = b.reference()
    keep = np.ones(got.shape[:2], bool)
    keep[rows, [3, 6]] = False
    with np.errstate(invalid="ignore"):
        ok = np.abs(got - ref) <= b.bound(ref, A, S)
    assert ok[keep].all() and np.array_equal(got[-rows:], good[-rows:])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attn_bad_pages_are_visible(dt):
    """A page outside the pool where keys are read: NaN for that sequence
    alone; a shared one: for all."""
    rows, lens = [2, 1, 3], [40, 70, 20]
    b = Batch8(dt, 4, 2, 64, 32, rows, lens, shared=40)
    good = f64(b.attend())
    b.d_table[1, 2] = b.k.shape[0]
    got = f64(b.attend())
    assert np.isnan(got[2]).all() and np.array_equal(np.delete(got, 2, 0), np.delete(good, 2, 0))
    b.d_shared[1] = -3
    assert np.isnan(f64(b.attend())).all()


def test_attn_plans_are_for_their_own_call():
    """A plan for other sizes, none, and one for a cache of 16 bits give NaN."""
    b, c = (Batch8("bf16", 4, 2, 64, 32, [1, 2], [40, 9], shared=s) for s in (20, 36))
    plan = torch.zeros(max(ooo.paged_plan8_bytes(x.batch) for x in (b, c)), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(ooo.paged_attn8_workspace(x.batch) for x in (b, c)), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(b.q)
    d = Batch("bf16", 4, 2, 64, 32, [1, 2], [40, 9], shared=20)
    for make in (lambda: plan, lambda: ooo.paged_plan8(c.batch, plan), lambda: ooo.paged_plan(d.batch, plan)):
        ooo.paged_attn8(b.batch, b.cache, make(), b.q, b.scale, out, ws)
        assert out.isnan().all()
    out.zero_()
    ooo.paged_attn(d.batch, ooo.paged_plan8(b.batch, plan), d.q, d.k, d.v, d.scale, out, ws)
    assert out.isnan().all()


def test_attn_bounds_device_values():
    b = Batch8("bf16", 4, 2, 64, 32, [2, 2], [10, 4], pad=1)
    b.d_len[0] = 1 << 29
    b.d_row_start[2] = 1 << 29
    out = b.attend()
    assert out.shape[0] == 5 and np.isnan(f64(out)[:2]).all()  # its table's unused entries are no pages
    b.d_row_start.copy_(torch.tensor([0, -5, -9], dtype=torch.int32))
    assert (f64(b.attend()) == 7.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_attn_same_bits_every_time(dt, D):
    other = torch.empty(1 << 26, device="cuda")
    for rows, lens, shared in (([2, 1, 3], [40, 50, 20], 20), ([1] * 9, [700] * 9, 0), ([90, 1, 33], [500, 90, 7], 300)):
        b = Batch8(dt, 4, 2, D, 32, rows, lens, shared=shared)
        first = b.attend()
        for _ in range(6):
            other.fill_(float("nan"))
            assert torch.equal(b.attend(), first)


def test_attn_pool_past_32_bits():
    """Pages, and scales, more than 2^32 bytes from the pool's start."""
    b = Batch8("bf16", 4, 2, 64, 32, [1, 3], [130, 90], shared=40)
    want = b.attend()
    page, n = 2 * 32 * 64, b.k.shape[0]
    stride = 900_000_000
    assert (n - 1) * stride > 1 << 32
    for x in ("k", "v"):
        big = torch.empty((n - 1) * stride + page, dtype=torch.uint8, device="cuda").as_strided(
            b.k.shape, (stride, 32 * 64, 64, 1))
        big.copy_(getattr(b, x))
        setattr(b, x, big)
        s = torch.empty((n - 1) * stride + 2, dtype=torch.uint8, device="cuda").as_strided(b.ks.shape, (stride, 1, 1))
        s.copy_(getattr(b, x + "s"))
        setattr(b, x + "s", s)
    b.bind()
    assert torch.equal(b.attend(), want)


@pytest.mark.parametrize("dt,shared", [("bf16", 0), ("bf16", 70), ("f32", 33)])
def test_attn_many_sequences(dt, shared):
    r = random.Random(5)
    lens = ragged(r, 700, 20)
    b = Batch8(dt, 4, 2, 64, 32, [1] * 699 + [35], lens, shared=shared, pad=1, seed=1)
    b.check(b.attend())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-40, -1e-40])
def test_attn_any_finite_scale(dt, D, scale):
    b = Batch8(dt, 4, 2, D, 32, [1, 40], [70, 300], shared=50)
    b.scale = scale
    b.check(b.attend())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 128)])
@pytest.mark.parametrize("exp", [-100, 60, 110])
def test_attn_scales_of_any_size(dt, D, exp):
    """V's scales from the least to the largest: outputs of their size."""
    b = Batch8(dt, 4, 2, D, 32, [1, 40], [70, 300], shared=50)
    b.vs.fill_(exp + 127)
    b.v.copy_(torch.randint(0, 0x58, b.v.shape, device="cuda"))  # up to 16
    b.check(b.attend())


def test_attn_layers():
    b = Batch8("bf16", 8, 2, 128, 32, [1, 40], [70, 200], shared=90, layers=3, gap=48, scale_gap=5)
    for layer in (2, 0, 1):
        got = f64(b.attend(layer=layer))
        ref, A, S = b.reference(layer)
        assert (np.abs(got - ref) <= b.bound(ref, A, S)).all()


def test_attn_two_batches_on_two_streams():
    bs = [Batch8("bf16", 8, 2, 128, 32, [1, 40, 3], [300, 90, 700], shared=200, seed=1),
          Batch8("bf16", 8, 2, 64, 32, [1] * 30, [100] * 30, shared=0, seed=2)]
    want = [b.attend() for b in bs]
    keep = [(ooo.paged_plan8(b.batch), torch.empty(ooo.paged_attn8_workspace(b.batch), dtype=torch.uint8,
                                                   device="cuda"), torch.full_like(b.q, 7.0)) for b in bs]
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in bs]
    for b, (plan, ws, out), s in zip(bs, keep, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ooo.paged_plan8(b.batch, plan)
            ooo.paged_attn8(b.batch, b.cache, plan, b.q, b.scale, out, ws)
        graphs.append(g)
    for _ in range(4):
        for _, _, out in keep:
            out.fill_(7.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (_, _, out), w in zip(keep, want):
            assert torch.equal(out, w)


# -------------------------------------------------------------- compaction


def random_paths(r, rows, extra=1):
    cap = max(max(rows), 1) + extra
    path, acc = np.full((len(rows), cap), -1, np.int32), np.zeros(len(rows), np.int32)
    for s, n in enumerate(rows):
        L = r.randint(-1, n - 1) if n else -1
        if L >= 0:
            path[s, :L + 1] = [0] + sorted(r.sample(range(1, n), L))
        acc[s] = L
    return path, acc


def check_compact(b, path, acc):
    want = [[oc.compact(c, s, b.row_start, b.lens, b.table, path, acc, b.page) for c, s in
             (zip(cs, ss) if cs.ndim == 5 else [(cs, ss)])] for cs, ss in b.bytes()]
    ooo.paged_compact8(b.batch, b.cache, torch.from_numpy(path).cuda(), torch.from_numpy(acc).cuda())
    for (cs, ss), w in zip(b.bytes(), want):
        cs, ss = (cs, ss) if cs.ndim == 5 else (cs[None], ss[None])
        for c, s, (wc, ws) in zip(cs, ss, w):
            assert np.array_equal(s, ws) and np.array_equal(c, wc)


@pytest.mark.parametrize("dt,D,layers,page,most", [("bf16", 128, 3, 32, 20), ("bf16", 64, 0, 64, 60),
                                                   ("f32", 64, 2, 32, 130), ("bf16", 128, 1, 128, 200)])
def test_compact(dt, D, layers, page, most):
    r = random.Random(most)
    rows, lens = ragged(r, 7, most), ragged(r, 7, 100)
    lens[1], lens[2] = 0, 32
    b = Batch8(dt, 4, 2, D, page, rows, lens, layers=layers, gap=32, scale_gap=2, seed=page, spread=2.0)
    check_compact(b, *random_paths(r, rows))


def test_compact_leaves_bad_entries():
    b = Batch8("bf16", 4, 2, 64, 32, [5, 40, 4, 6, 3], [30, 0, 31, 7, 9])
    path = np.array([[0, 3, 9], [0, 35, 38], [0, 1, 2], [-1, 2, 4], [0, 1, 2]], np.int32)
    acc = np.array([2, 2, 7, 2, -1], np.int32)  # row 9 is none of five; 7 is past path_cap; -1
    check_compact(b, path, acc)
    before = b.bytes()
    b.d_table[1, 1] = -1   # rows 35 and 38 lie nowhere
    b.d_len[3] = -2
    b.d_len[4] = 1 << 30
    ooo.paged_compact8(b.batch, b.cache, torch.tensor([[0, 35, 38]] * 5, dtype=torch.int32, device="cuda"),
                       torch.full((5,), 2, dtype=torch.int32, device="cuda"))
    for (c0, s0), (c1, s1) in zip(before, b.bytes()):
        assert np.array_equal(c0, c1) and np.array_equal(s0, s1)


# -------------------------------------------------------------------- fork


class Forks:
    """A pool of any type with parents' tables and children's pages."""

    def __init__(self, kind, lens, page, layers=2, Hkv=2, D=64, gap=0, seed=0):
        r = np.random.default_rng(seed)
        n = len(lens)
        self.kind, self.page, self.lens = kind, page, list(lens)
        ld = max(m // page for m in lens) + 2
        pages = n * ld + n + 1
        ids = r.permutation(pages).astype(np.int32)
        self.table = ids[:n * ld].reshape(n, ld).copy()
        self.fresh = ids[n * ld:n * ld + n].copy()
        dt = {"f8": torch.uint8, "bf16": torch.bfloat16, "f32": torch.float32}[kind]
        g = torch.Generator(device="cuda").manual_seed(seed)
        size = Hkv * page * D

        def pool(width, inner):
            t = torch.randint(0, 100, (layers, pages, width + gap), generator=g, device="cuda").to(dt)
            return t[..., :width].unflatten(-1, inner)
        self.pools = [pool(size, (Hkv, page, D)) for _ in range(2)]
        self.scales = [pool(Hkv * page // 32, (Hkv, page // 32)) for _ in range(2)] if kind == "f8" else []
        self.d_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.d_table = torch.from_numpy(self.table).cuda()
        row_start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        f8 = torch.float8_e4m3fn
        first = self.pools[0][0].view(f8) if kind == "f8" else self.pools[0][0]
        more = {"dtype": torch.bfloat16} if kind == "f8" else {}
        self.batch = ooo.PagedBatch(row_start, self.d_len, self.d_table, first, Hkv, 1, **more)
        if kind == "f8":
            self.cache = ooo.Cache8(self.batch, *(p.view(f8) for p in self.pools), *self.scales)

    def call(self, parent, fresh, lens, table, stream=None):
        p, f = (torch.from_numpy(np.asarray(t, np.int32)).cuda() for t in (parent, fresh))
        if self.kind == "f8":
            ooo.paged_fork8(self.batch, self.cache, p, f, lens, table, stream=stream)
        else:
            ooo.paged_fork(self.batch, *self.pools, p, f, lens, table, stream=stream)

    def check(self, parent, in_place, fresh=None):
        fresh = self.fresh if fresh is None else fresh
        want_n, want_t, copies = oc.fork(self.lens, self.table, parent, fresh, self.pools[0].shape[1], self.page,
                                         in_place)
        want = [t.float().cpu().numpy().copy() for t in (*self.pools, *self.scales)]
        for t in want:
            old = t.copy()
            for _, src, dst, rows in copies:
                n = rows if t.ndim == 5 else (rows + 31) // 32
                t[:, dst, :, :n] = old[:, src, :, :n]
        lens, table = (self.d_len, self.d_table) if in_place else (
            torch.full_like(self.d_len, -9), torch.full_like(self.d_table, -9))
        self.call(parent, fresh, lens, table)
        assert lens.tolist() == want_n.tolist() and np.array_equal(table.cpu().numpy(), want_t)
        for t, w in zip((*self.pools, *self.scales), want):
            assert np.array_equal(t.float().cpu().numpy(), w)
        if not in_place:
            assert self.d_len.tolist() == self.lens and np.array_equal(self.d_table.cpu().numpy(), self.table)
        return copies


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind,page,Hkv,D", [("f8", 32, 2, 64), ("f8", 128, 3, 128), ("bf16", 16, 1, 128),
                                             ("bf16", 64, 2, 64), ("f32", 16, 2, 64), ("f32", 128, 1, 128)])
def test_fork(kind, page, Hkv, D, in_place):
    lens = [0, 1, page - 1, page, page + 1, 3 * page + 5, 33, 5, 9, 2]
    f = Forks(kind, lens, page, Hkv=Hkv, D=D, gap=16, seed=page)
    assert len(f.check([-1, 5, 5, 0, 5, -1, 6, 4, 3, -1], in_place)) == 3 + (not in_place)


def test_fork_beams_change_places():
    f = Forks("f8", [40, 7, 64, 33], 32)
    assert len(f.check([1, 0, 3, 0], False)) == 4
    f = Forks("bf16", [40, 7, 64, 33], 16)
    assert len(f.check([1, 0, 3, 0], True)) == 0  # every parent has a parent


@pytest.mark.parametrize("kind", ["f8", "f32"])
def test_fork_leaves_what_it_cannot_do(kind):
    f = Forks(kind, [40, 7, 64, 33, 20, 3], 32)
    fresh = f.fresh.copy()
    fresh[1], fresh[2] = -1, f.pools[0].shape[1]
    f.table[5, 0] = 1 << 20  # the parent's open page is none
    f.d_table.copy_(torch.from_numpy(f.table))
    assert len(f.check([-1, 0, 0, 6, 5, -1], True, fresh)) == 0
    f.lens[0] = f.table.shape[1] * 32  # fills its table
    f.lens[1] = -1
    f.d_len.copy_(torch.tensor(f.lens, dtype=torch.int32))
    assert len(f.check([-1, -1, 0, 1, -1, -1], True)) == 0
    f.check([-1, -1, 0, 1, -1, -1], False)


def test_fork_refuses_half_in_place_and_overlaps():
    f = Forks("bf16", [40, 7], 16)
    with pytest.raises(ooo.OooError, match="both"):
        f.call([-1, 0], f.fresh, f.d_len, f.d_table.clone())
    both = torch.zeros(5, dtype=torch.int32, device="cuda")
    g = Forks("bf16", [40, 7], 16)
    g.batch.struct.seq_len = both.data_ptr()
    with pytest.raises(ValueError, match="overlaps"):
        g.call([-1, 0], g.fresh, both[1:3], g.d_table.clone())


# --------------------------------------------------------- Python's refusals


def test_python_refusals():
    f8 = torch.float8_e4m3fn
    b = Batch8("bf16", 4, 2, 64, 32, [1, 2], [40, 9], layers=2)
    d = Batch("bf16", 4, 2, 64, 32, [1, 2], [40, 9])
    k, v = b.k.view(f8), b.v.view(f8)
    pages = k[0]
    make = lambda **kw: ooo.PagedBatch(b.d_row_start, b.d_len, b.d_table, pages, 4, b.n_rows, **kw)  # noqa: E731
    with pytest.raises(ValueError, match="dtype"):
        make()
    with pytest.raises(ValueError, match="dtype"):
        make(dtype=torch.float16)
    with pytest.raises(ValueError, match="dtype"):
        ooo.PagedBatch(b.d_row_start, b.d_len, b.d_table, d.k, 4, b.n_rows, dtype=torch.float32)
    with pytest.raises(ValueError, match="not float8"):
        ooo.Cache8(d.batch, k, v, b.ks, b.vs)
    for args in ((k, v[:1], b.ks, b.vs), (k, v, b.ks[:, :-1], b.vs), (k, v, b.ks.int(), b.vs), (b.k, v, b.ks, b.vs),
                 (k, v, b.ks.cpu(), b.vs)):
        with pytest.raises(ValueError):
            ooo.Cache8(b.batch, *args)
    c = Batch8("bf16", 4, 2, 64, 64, [1, 2], [40, 9])
    with pytest.raises(ValueError, match="contiguous"):
        ooo.Cache8(c.batch, c.k.view(f8), c.v.view(f8), c.ks.transpose(1, 2).contiguous().transpose(1, 2), c.vs)
    wide = torch.zeros((*b.ks.shape[:2], 7), dtype=torch.uint8, device="cuda")[..., :2].unflatten(-1, (2, 1))
    with pytest.raises(ValueError, match="same strides"):
        ooo.Cache8(b.batch, k, v, wide, b.vs)
    with pytest.raises(ValueError, match="not for this call"):
        ooo.paged_plan8(d.batch)
    with pytest.raises(ValueError, match="not for this call"):
        ooo.paged_attn(b.batch, torch.zeros(16, dtype=torch.uint8, device="cuda"), b.q, pages, pages, 1.0, b.q,
                       torch.zeros(16, device="cuda"))
    with pytest.raises(ValueError, match="other pages"):
        ooo.paged_compact8(c.batch, b.cache, torch.zeros((2, 4), dtype=torch.int32, device="cuda"), c.d_len)
    with pytest.raises(ooo.OooError, match="layer"):
        b.attend(layer=2)


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_steps_captured_and_replayed(dt):
    """A step as a serving loop has it, captured and replayed while lengths and
    tables grow: append, plan, attention, compaction, then a fork of two
    sequences; each replay against the same calls made one by one, and its
    parts against the reference."""
    r = random.Random(11)
    rows, lens = [4, 1, 36, 3], [30, 14, 0, 77]
    mask = bh.trie_masks(r, rows, 1)[0]
    a, e = (Batch8(dt, 8, 2, 64, 32, rows, lens, shared=50, mask=mask, pad=2, seed=5, spare=60, table_pad=6)
            for _ in range(2))
    r2 = np.random.default_rng(3)
    used = set(a.shared_ids.tolist()) | {int(x) for row in a.table for x in row if x >= 0}
    free = [p for p in r2.permutation(a.k.shape[0]).tolist() if p not in used]
    for s in range(4):
        for t in range(a.table.shape[1]):
            if a.table[s, t] < 0:
                a.table[s, t] = free.pop()
    for b in (a, e):
        b.table = a.table.copy()
        b.d_table.copy_(torch.from_numpy(a.table))
    depth = torch.from_numpy(np.concatenate([bh.trie_masks(random.Random(11), rows, 1)[1],
                                             np.zeros(2, np.int32)])).cuda()
    width = (8 + 4) * 64

    def buffers(b):
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        return {"qkv": torch.zeros((b.n_rows, width), dtype=b.dt, device="cuda"), "q": torch.full_like(b.q, 7.0),
                "out": torch.full_like(b.q, 7.0), "path": i32(4, 37), "acc": i32(4), "parent": i32(4),
                "fresh": i32(4), "plan": torch.zeros(ooo.paged_plan8_bytes(b.batch), dtype=torch.uint8, device="cuda"),
                "ws": torch.full((ooo.paged_attn8_workspace(b.batch),), 0xFF, dtype=torch.uint8, device="cuda")}

    def step(b, t):
        ooo.paged_append8(b.batch, b.cache, t["qkv"], None, None, 1e-6, 1e6, t["q"], depth=depth)
        ooo.paged_plan8(b.batch, t["plan"])
        ooo.paged_attn8(b.batch, b.cache, t["plan"], t["q"], b.scale, t["out"], t["ws"])
        ooo.paged_compact8(b.batch, b.cache, t["path"], t["acc"])
        b.d_len.add_(t["acc"] + 1)

    def fork(b, t):
        ooo.paged_fork8(b.batch, b.cache, t["parent"], t["fresh"], b.d_len, b.d_table)

    ta, te = buffers(a), buffers(e)
    start = [x.clone() for x in (a.k, a.v, a.ks, a.vs, a.d_len, a.d_table)]
    step(a, ta)
    fork(a, ta)
    for x, y in zip((a.k, a.v, a.ks, a.vs, a.d_len, a.d_table), start):
        x.copy_(y)
    torch.cuda.synchronize()
    stream, graphs = torch.cuda.Stream(), []
    for f in (step, fork):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            f(a, ta)
        graphs.append(g)
    for n in range(5):
        gen = torch.Generator(device="cuda").manual_seed(100 + n)
        qkv = (torch.randn((a.n_rows, width), generator=gen, device="cuda") * (1 + n)).to(a.dt)
        path, acc = np.full((4, 37), -1, np.int32), np.zeros(4, np.int32)
        for s, m in enumerate(rows):
            node = r.randrange(m)
            p = [j for j in range(m) if (int(mask[a.row_start[s] + node, 0]) >> j) & 1]
            path[s, :len(p)], acc[s] = p, len(p) - 1
        parent = np.full(4, -1, np.int32)
        kids = [(0, 3), (1, 2)] if n % 2 == 0 else [(2, 0)]
        for child, par in kids:
            parent[child] = par
        fresh = np.array([free.pop() if p >= 0 else -1 for p in parent], np.int32)
        for t in (ta, te):
            t["qkv"].copy_(qkv)
            for k, x in (("path", path), ("acc", acc), ("parent", parent), ("fresh", fresh)):
                t[k].copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        graphs[0].replay()
        step(e, te)
        torch.cuda.synchronize()
        assert torch.equal(ta["out"], te["out"]) and torch.equal(ta["q"], te["q"])
        for x in ("k", "v", "ks", "vs", "d_len"):
            assert torch.equal(getattr(a, x), getattr(e, x))
        a.lens = a.d_len.tolist()
        want_n, want_t, _ = oc.fork(a.lens, a.table, parent, fresh, a.k.shape[0], 32, True)
        graphs[1].replay()
        fork(e, te)
        torch.cuda.synchronize()
        for x in ("k", "v", "ks", "vs", "d_len", "d_table"):
            assert torch.equal(getattr(a, x), getattr(e, x))
        assert a.d_len.tolist() == want_n.tolist() and np.array_equal(a.d_table.cpu().numpy(), want_t)
        a.lens, a.table = want_n.tolist(), want_t
        # every sequence's cache as it is now, a child's over its parent's pages and its own
        one = Batch8(dt, 8, 2, 64, 32, [1] * 4, [m - 1 for m in a.lens], shared=0, spare=60)
        one.k, one.v, one.ks, one.vs = a.k, a.v, a.ks, a.vs
        one.d_table, one.table = a.d_table, a.table
        one.bind()
        one.q[:] = one.q[:1]
        one.check(one.attend())
