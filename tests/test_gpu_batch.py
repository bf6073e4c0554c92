"""The batch's entry points on the GPU against the float64 reference."""

import math
import random

import numpy as np
import pytest
import torch

from oracle import batch as ob
from paper_2608_00814_amd import ooo

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import batch_harness as bh
    from batch_harness import HALF, TYPES, U32, Batch, ragged


def f64(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------ append


def run_append(b, norm, depth, seed=1, ld_gap=0, theta=1e6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (b.Hq + 2 * b.Hkv) * b.D
    qkv = torch.randn((b.n_rows, width + ld_gap), generator=g, device="cuda").to(b.dt)[:, :width]
    qw, kw = ((torch.randn(b.D, generator=g, device="cuda") * 0.1 + 1).to(b.dt) if norm else None for _ in range(2))
    d = None if depth is None else torch.from_numpy(depth).cuda()
    q_out = torch.full((b.n_rows, b.Hq, b.D), 7.0, dtype=b.dt, device="cuda")
    k0, v0 = f64(b.k), f64(b.v)
    ooo.paged_append(b.batch, qkv, qw, kw, 1e-6, theta, q_out, b.k, b.v, depth=d)
    got_q, got_k, got_v = f64(q_out), f64(b.k), f64(b.v)
    h = HALF[b.kind]
    x = f64(qkv)
    nq, nk = (None, None) if not norm else (f64(qw), f64(kw))
    assert (got_q[b.total:] == 7.0).all()
    for s in range(len(b.rows)):
        for i in range(b.rows[s]):
            r = b.row_start[s] + i
            pos = b.shared + b.lens[s] + (i if depth is None else int(depth[r]))
            q, k, v, sq, sk = ob.append_row(x[r], pos, b.Hq, b.Hkv, b.D, nq, nk, 1e-6, theta)
            pg, sl = ob.place(b.table[s], b.lens[s] + i, b.page)
            # half a step of the stored value; norm factor, sine and cosine
            # and two products in float32: under 64 roundings of the pair
            assert (np.abs(got_q[r] - q) <= h * np.abs(q) + 64 * U32 * sq).all(), (s, i)
            assert (np.abs(got_k[pg, :, sl] - k) <= h * np.abs(k) + 64 * U32 * sk).all(), (s, i)
            assert np.array_equal(got_v[pg, :, sl], v)
            k0[pg, :, sl], v0[pg, :, sl] = got_k[pg, :, sl], got_v[pg, :, sl]
    assert np.array_equal(k0, got_k) and np.array_equal(v0, got_v), "rows of other places were written"


@pytest.mark.parametrize("dt,Hq,Hkv,D,page,norm,trie", [
    ("bf16", 32, 8, 128, 64, True, False), ("bf16", 40, 8, 128, 16, True, True), ("bf16", 14, 2, 64, 32, False, False),
    ("bf16", 3, 1, 128, 128, True, False), ("f32", 4, 1, 64, 16, True, True), ("f32", 16, 8, 128, 32, False, False),
    ("f32", 5, 5, 128, 16, True, False),
])
def test_append(dt, Hq, Hkv, D, page, norm, trie):
    r = random.Random(3)
    rows = ragged(r, 9, 21)
    rows[0] = rows[4] = 0
    lens = ragged(r, 9, 150)
    depth = None
    if trie:
        depth = np.concatenate([bh.trie_masks(r, rows, 1)[1], np.full(3, 99, np.int32)])
    run_append(Batch(dt, Hq, Hkv, D, page, rows, lens, shared=77, pad=3, gap=64), norm, depth, ld_gap=16)


def test_append_far_position_and_one_row():
    run_append(Batch("f32", 2, 1, 64, 16, [1], [0], shared=900000), True, None)
    run_append(Batch("bf16", 4, 2, 64, 16, [1], [3], shared=0), True, None, theta=1e4)


def test_append_many_sequences():
    r = random.Random(5)
    run_append(Batch("bf16", 2, 1, 64, 16, ragged(r, 300, 2), ragged(r, 300, 40), shared=5), False, None)


def test_append_drops_rows_without_a_page():
    b = Batch("bf16", 8, 2, 64, 16, [20, 8, 4], [0, 14, 5])
    b.table[1, 1] = b.k.shape[0]  # one past the pool
    b.table[2, 0] = -1
    b.d_table.copy_(torch.from_numpy(b.table))
    b.d_len[0] = 2 ** 30          # past its table
    width = 12 * 64
    qkv = torch.randn((b.n_rows, width), device="cuda").to(b.dt)
    q_out = torch.full((b.n_rows, 8, 64), 7.0, dtype=b.dt, device="cuda")
    k0 = f64(b.k)
    ooo.paged_append(b.batch, qkv, None, None, 1e-6, 1e6, q_out, b.k, b.v)
    got, diff = f64(b.k), np.argwhere((f64(b.k) != k0).any(axis=(1, 3)))
    pg, sl = ob.place(b.table[1], 14, 16), ob.place(b.table[1], 15, 16)
    assert {tuple(d) for d in diff} == {pg, sl}  # the two rows of sequence 1 on its good page
    assert not (f64(q_out) == 7.0).all(axis=2).any()
    assert np.isfinite(got).all()


@pytest.mark.parametrize("starts", [[5, 9, 14], [0, 9, 4], [9, -3, 14], [-4, 9, 1 << 30]])
def test_append_bounds_row_starts(starts):
    """row_start that does not begin at 0 or falls: rows outside every
    sequence's range have no place (none ahead of a page table either)."""
    b = Batch("bf16", 2, 1, 64, 16, [9, 5], [0, 0])
    b.d_row_start.copy_(torch.tensor(starts, dtype=torch.int32))
    qkv = torch.randn((b.n_rows, 4 * 64), device="cuda").to(b.dt)
    q_out = torch.full((b.n_rows, 2, 64), 7.0, dtype=b.dt, device="cuda")
    k0, v0 = f64(b.k), f64(b.v)
    ooo.paged_append(b.batch, qkv, None, None, 1e-6, 1e6, q_out, b.k, b.v)
    R = min(max(starts[2], 0), b.n_rows)
    lo = [min(max(s, 0), R) for s in starts]
    places = set()
    for s in range(2):
        places |= {ob.place(b.table[s], i, 16) for i in range(min(max(starts[s + 1], lo[s]), R) - lo[s])}
    got = {tuple(d) for d in np.argwhere((f64(b.v) != v0).any(axis=(1, 3)))}
    assert got <= places and {tuple(d) for d in np.argwhere((f64(b.k) != k0).any(axis=(1, 3)))} <= places
    if starts[0] == 5:  # two sequences of 4 and 5 rows behind 5 that are none's
        assert got == places and (f64(q_out)[:5] == 7.0).all() and not (f64(q_out)[5:] == 7.0).all(axis=2).any()
    assert (f64(q_out)[R:] == 7.0).all()


# --------------------------------------------------------------- attention


@pytest.mark.parametrize("shared", [0, 1, 63, 64, 200])
@pytest.mark.parametrize("dt,Hq,Hkv,D,page", [
    ("bf16", 8, 2, 128, 16), ("bf16", 14, 2, 64, 64), ("bf16", 5, 1, 128, 32), ("f32", 4, 1, 64, 16),
    ("f32", 6, 2, 128, 128),
])
def test_attn_decode(dt, Hq, Hkv, D, page, shared):
    r = random.Random(shared)
    lens = [0, 1, 15, 16, 63, 64, 65] + ragged(r, 4, 200)
    Batch_ = Batch(dt, Hq, Hkv, D, page, [1] * len(lens), lens, shared=shared, pad=2, seed=shared)
    Batch_.check(Batch_.attend())


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
    b = Batch(dt, Hq, Hkv, D, 16, rows, lens, shared=shared, mask=mask, pad=3, seed=most, gap=32)
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
    b = Batch(dt, 4, 2, 64, 16, rows, lens, shared=shared, mask=mask, seed=9)
    out = b.attend()
    b.check(out)
    if shared == 0:
        assert not out[3].any() and not out[33].any()


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attn_long_splits(dt, D):
    """Long own caches and a long prompt: many parts to join."""
    for rows, lens, shared in (([1], [3000], 0), ([1, 2], [1500, 10], 2100), ([40, 1], [700, 2000], 900)):
        b = Batch(dt, 8, 2, D, 64, rows, lens, shared=shared, seed=lens[0])
        b.check(b.attend())


def test_attn_wide_prompt_chunk():
    b = Batch("bf16", 4, 1, 128, 32, [150, 300], [33, 0], shared=40)
    b.check(b.attend())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_attn_what_is_not_seen_does_not_matter(dt, D):
    """NaN and infinities in unused slots and in new rows that a row does not
    see leave it as it is; the rows that see them are not finite."""
    r = random.Random(1)
    rows, lens = [12, 40, 1], [10, 77, 64]
    mask = bh.trie_masks(r, rows, 1)[0]
    b = Batch(dt, 8, 2, D, 16, rows, lens, shared=30, mask=mask, seed=4)
    for s, (n, m) in enumerate(zip(rows, lens)):  # behind each sequence's end
        for t in range(n + m, (n + m + 15) // 16 * 16):
            pg, sl = ob.place(b.table[s], t, 16)
            b.k[pg, :, sl], b.v[pg, :, sl] = float("nan"), float("inf")
    for t in range(30, 32):
        pg, sl = ob.place(b.shared_ids, t, 16)
        b.k[pg, :, sl], b.v[pg, :, sl] = float("inf"), float("nan")
    b.check(b.attend())
    for j, bad in ((5, float("inf")), (30, float("nan")), (39, float("-inf"))):
        pg, sl = ob.place(b.table[1], 77 + j, 16)
        b.v[pg, :, sl] = bad
        if j == 30:
            b.k[pg, :, sl] = bad
    out = b.attend()
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
def test_attn_bad_pages_are_visible(dt):
    """A page outside the pool where keys are read: NaN for that sequence
    alone; a shared one: for all."""
    rows, lens = [2, 1, 3], [40, 50, 20]
    b = Batch(dt, 4, 2, 64, 16, rows, lens, shared=20)
    good = f64(b.attend())
    b.d_table[1, 2] = b.k.shape[0]
    got = f64(b.attend())
    assert np.isnan(got[2]).all() and np.array_equal(np.delete(got, 2, 0), np.delete(good, 2, 0))
    b.d_shared[1] = -3
    assert np.isnan(f64(b.attend())).all()


def test_attn_plan_of_other_sizes_gives_nan():
    b, c = (Batch("bf16", 4, 2, 64, 16, [1, 2], [40, 9], shared=s) for s in (20, 36))
    plan = torch.zeros(max(ooo.paged_plan_bytes(x.batch) for x in (b, c)), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(ooo.paged_attn_workspace(x.batch) for x in (b, c)), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(b.q)
    for p in (plan, ooo.paged_plan(c.batch, plan)):  # never made, made for another prompt
        ooo.paged_attn(b.batch, p, b.q, b.k, b.v, b.scale, out, ws)
        assert out.isnan().all()


def test_attn_bounds_device_values():
    """Lengths and row counts past what buffers and tables hold are cut."""
    b = Batch("bf16", 4, 2, 64, 16, [2, 2], [10, 4], pad=1)
    b.d_len[0] = 1 << 29
    b.d_row_start[2] = 1 << 29
    out = b.attend()
    assert out.shape[0] == 5 and np.isnan(f64(out)[:2]).all()  # its table's unused entries are no pages
    b.d_row_start.copy_(torch.tensor([0, -5, -9], dtype=torch.int32))
    assert (f64(b.attend()) == 7.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_attn_same_bits_every_time(dt, D):
    """Short and long items of both kinds, with other work in between."""
    other = torch.empty(1 << 26, device="cuda")
    for rows, lens, shared in (([2, 1, 3], [40, 50, 20], 20), ([1] * 9, [700] * 9, 0), ([90, 1, 33], [500, 90, 7], 300)):
        b = Batch(dt, 4, 2, D, 16, rows, lens, shared=shared)
        first = b.attend()
        for _ in range(6):
            other.fill_(float("nan"))
            assert torch.equal(b.attend(), first)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attn_deterministic_and_on_a_stream(dt):
    b = Batch(dt, 8, 2, 128, 32, [1, 5, 40], [500, 90, 7], shared=300)
    a = b.attend()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = b.attend()
    s.synchronize()
    d = b.attend(stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(a, c) and torch.equal(a, d)


def test_attn_pool_past_32_bits():
    """Pages more than 2^32 elements from the pool's start."""
    b = Batch("bf16", 4, 2, 64, 16, [1, 3], [30, 20], shared=17)
    want = b.attend()
    page = 2 * 16 * 64
    stride = 900_000_000
    n = b.k.shape[0]
    big = []
    for t in (b.k, b.v):
        p = torch.empty((n - 1) * stride + page, dtype=b.dt, device="cuda").as_strided(
            t.shape, (stride, 16 * 64, 64, 1))
        p.copy_(t)
        big.append(p)
    assert (n - 1) * stride > 1 << 32
    b.k, b.v = big
    b.batch = ooo.PagedBatch(b.d_row_start, b.d_len, b.d_table, b.k, 4, b.n_rows, shared_pages=b.d_shared,
                             shared_len=17)
    assert torch.equal(b.attend(), want)


@pytest.mark.parametrize("dt,shared", [("bf16", 0), ("bf16", 70), ("f32", 33)])
def test_attn_many_sequences(dt, shared):
    r = random.Random(5)
    lens = ragged(r, 700, 20)
    b = Batch(dt, 4, 2, 64, 16, [1] * 699 + [35], lens, shared=shared, pad=1, seed=1)
    b.check(b.attend())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("shared", [0, 2601, 4096])
def test_attn_many_pages(dt, D, shared):
    """Hundreds of the smallest pages to a part, in both kinds of it."""
    for rows, lens in (([1, 2], [5003, 3]), ([70, 1], [2100, 4100])):
        b = Batch(dt, 2, 1, D, 16, rows, lens, shared=shared, seed=shared)
        b.check(b.attend())


@pytest.mark.parametrize("dt,heads", [("bf16", 100), ("bf16", 256), ("f32", 300)])
def test_attn_more_heads_than_work_is_shared_over(dt, heads):
    for shared in (0, 50):
        b = Batch(dt, heads, heads, 64, 16, [1, 40, 2], [30, 70, 5], shared=shared, pad=1, seed=heads)
        b.check(b.attend())


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("shared,page", [(0, 16), (333, 32), (1000, 128)])
def test_attn_tries_over_long_sequences(dt, D, shared, page):
    """Many rows with masks behind more keys than a short block has; masks that
    begin inside a tile, blocks whose last rows are few."""
    r = random.Random(D)
    rows, lens = [64, 3, 150, 40, 33], [300, 700, 261, 1000, 321]
    mask = bh.trie_masks(r, rows, 3)[0]
    b = Batch(dt, 8, 2, D, page, rows, lens, shared=shared, mask=mask, pad=1, seed=shared)
    b.check(b.attend())
    c = Batch(dt, 8, 2, D, page, rows, lens, shared=shared, seed=shared + 1)
    c.check(c.attend())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_attn_what_is_not_seen_behind_long_sequences(dt, D):
    r = random.Random(2)
    rows, lens, shared = [90, 34], [300, 417], 410
    mask = bh.trie_masks(r, rows, 2)[0]
    b = Batch(dt, 8, 2, D, 16, rows, lens, shared=shared, mask=mask, seed=4)
    for ids, n in ((b.table[0], 390), (b.table[1], 451), (b.shared_ids, shared)):
        for t in range(n, (n + 15) // 16 * 16):
            pg, sl = ob.place(ids, t, 16)
            b.k[pg, :, sl], b.v[pg, :, sl] = float("nan"), float("inf")
    b.check(b.attend())
    for j, bad in ((7, float("inf")), (66, float("nan")), (89, float("-inf"))):
        pg, sl = ob.place(b.table[0], 300 + j, 16)
        b.v[pg, :, sl] = bad
        if j == 66:
            b.k[pg, :, sl] = bad
    got = f64(b.attend())
    ref, A, S = b.reference()
    hit = np.zeros(b.total, bool)
    hit[:90] = np.array([[(int(mask[x, j // 64]) >> (j % 64)) & 1 for j in (7, 66, 89)] for x in range(90)]).any(axis=1)
    assert hit[:90].any() and not hit[:90].all()
    assert not np.isfinite(got[hit]).any(), "a seen value that is not finite was lost"
    with np.errstate(invalid="ignore"):
        err, lim = np.abs(got[~hit] - ref[~hit]), b.bound(ref, A, S)[~hit]
    assert (err <= lim).all()


def test_attn_bad_pages_of_long_sequences_are_visible():
    b = Batch("bf16", 4, 2, 128, 16, [40, 1, 50], [600, 40, 900], shared=700)
    good = f64(b.attend())
    b.d_table[2, 30] = -1
    got = f64(b.attend())
    assert np.isnan(got[41:]).all() and np.array_equal(got[:41], good[:41])
    b.d_shared[20] = b.k.shape[0]
    assert np.isnan(f64(b.attend())).all()


def test_attn_two_batches_on_two_streams():
    """Captured together and replayed, each with its own plan and workspace."""
    bs = [Batch("bf16", 8, 2, 128, 16, rows, lens, shared=sh, seed=sh)
          for rows, lens, sh in (([1] * 6, [900, 40, 300, 0, 64, 5], 500), ([40, 3], [700, 90], 65))]
    want = [b.attend() for b in bs]
    keep = [(ooo.paged_plan(b.batch), torch.empty(ooo.paged_attn_workspace(b.batch), dtype=torch.uint8, device="cuda"),
             torch.empty_like(b.q)) for b in bs]
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in bs]
    for b, (plan, ws, out), s in zip(bs, keep, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ooo.paged_plan(b.batch, plan)
            ooo.paged_attn(b.batch, plan, b.q, b.k, b.v, b.scale, out, ws)
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,lens,shared", [([1, 2], [500, 64], 0), ([1] * 5, [200, 31, 0, 96, 33], 320),
                                              ([60, 40], [300, 416], 0), ([64], [512], 640)])
def test_attn_weights_sum_to_one(D, rows, lens, shared):
    """Where all keys have the same v it comes out unchanged, however the
    probabilities were rounded: numerator and denominator hold the same ones.
    Every 32nd key scores 0, the others' probabilities lie 0.0035 of themselves
    above a bf16 value, all to one side; v lies just below 2, where half a step
    is 0.00196 of it.  What is left are float32 roundings, under 3 (n + 64) of
    them of 2^-24 each (sums of n terms in O and in l, factors between parts):
    0.0002 at n = 1152."""
    b = Batch("bf16", 8, 2, D, 16, rows, lens, shared=shared)
    b.scale = -math.log(0.50175)  # a key of -1 gets exp(-scale) = 0.50175 of a key of 0
    b.q.zero_()
    b.q[..., 0] = 1
    b.k.zero_()
    for ids, n in [(b.shared_ids, shared)] + [(t, n + m) for t, n, m in zip(b.table, b.rows, b.lens)]:
        for t in range(n):
            pg, sl = ob.place(ids, t, 16)
            b.k[pg, :, sl, 0] = 0 if t % 32 == 0 else -1
    c = torch.tensor([1.9921875, -1.984375, 0.99609375, -3.984375], device="cuda").repeat(D // 4).to(b.dt)
    b.v.copy_(c.expand_as(b.v))
    out = b.attend()
    assert torch.equal(out[:b.total], c.expand(b.total, 8, D))


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("scale", [0.0, -0.0, -0.125, 1e-40, -1e-40])
def test_attn_any_finite_scale(dt, D, scale):
    """Zero weighs all seen keys alike, a negative one prefers the least
    products; short last tiles, masks and parts among narrow and wide blocks."""
    r = random.Random(D)
    for rows, lens, shared in (([1, 3], [70, 5], 0), ([1, 2, 5], [600, 33, 0], 90), ([50, 34], [290, 417], 0),
                               ([64], [300], 333)):
        for mask in (None, bh.trie_masks(r, rows, 1)[0]):
            b = Batch(dt, 8, 2, D, 16, rows, lens, shared=shared, mask=mask, pad=1, seed=shared)
            b.scale = scale
            b.check(b.attend())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [0, 40])
def test_attn_row_starts_that_fall_are_visible(dt, shared):
    """Sequences that would overlap: NaN rows, and a plan of no work."""
    b = Batch(dt, 4, 2, 64, 16, [30, 5, 1], [40, 9, 70], shared=shared, pad=2)
    good = b.attend()
    for starts in ([0, 30, 10, 36], [36, 0, 36, 36], [3, 30, 29, 36]):
        b.d_row_start.copy_(torch.tensor(starts, dtype=torch.int32))
        out = b.attend()
        assert out[:36].isnan().all() and (out[36:] == 7.0).all()
    b.d_row_start.copy_(torch.tensor([0, 30, 35, 36], dtype=torch.int32))
    assert torch.equal(b.attend(), good)


def test_attn_row_starts_past_the_buffers():
    """Cut to n_rows; rows ahead of row_start[0] are no sequence's and stay as
    they are."""
    b = Batch("bf16", 4, 2, 64, 16, [30, 5, 1], [40, 9, 70])
    good = b.attend()
    b.d_row_start.copy_(torch.tensor([0, 30, 35, 1 << 30], dtype=torch.int32))
    assert torch.equal(b.attend(), good)
    b.d_row_start.copy_(torch.tensor([3, 30, 35, 36], dtype=torch.int32))
    out = b.attend()
    assert (out[:3] == 7.0).all() and torch.equal(out[30:], good[30:]) and out[3:30].isfinite().all()


def batch_us(b, plan, ws, out):
    """Least of ten calls."""
    e = [torch.cuda.Event(enable_timing=True) for _ in range(11)]
    for x in e:
        x.record()
        ooo.paged_attn(b.batch, plan, b.q, b.k, b.v, b.scale, out, ws)
    torch.cuda.synchronize()
    return 1e3 * min(x.elapsed_time(y) for x, y in zip(e, e[1:]))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 20])
def test_attn_bad_queries_stay_their_own(dt, rows):
    """Queries and keys that are not finite: NaN rows for their sequence, the
    same bits for the others, and no second pass over the shared keys (40 times
    the batch's time; 4 leaves room for noise)."""
    n = 40 // rows
    b = Batch(dt, 8, 2, 128, 16, [rows] * n, [50] * n, shared=2000, pad=1, seed=rows)
    plan, out = ooo.paged_plan(b.batch), torch.full_like(b.q, 7.0)
    ws = torch.empty(ooo.paged_attn_workspace(b.batch), dtype=torch.uint8, device="cuda")
    good, before = b.attend(), batch_us(b, plan, ws, out)
    b.q[rows:2 * rows, 3, 5] = float("nan")      # a query head of sequence 1
    b.q[0, 1] = float("inf")
    pg, sl = ob.place(b.table[n - 1], 7, 16)
    b.k[pg, 1, sl] = float("nan")                # a key of the last sequence's second KV head
    after = batch_us(b, plan, ws, out)
    bad = torch.zeros(b.n_rows, 8, dtype=torch.bool, device="cuda")
    bad[rows:2 * rows, 3] = bad[0, 1] = True
    bad[b.total - rows:b.total, 4:] = True
    assert out[bad].isnan().all() and torch.equal(out[~bad], good[~bad])
    assert after < 4 * before, (before, after)


# ----------------------------------------------------------------- compact


@pytest.mark.parametrize("dt,D,layers,page", [("bf16", 128, 3, 16), ("bf16", 64, 1, 64), ("f32", 64, 2, 16),
                                              ("f32", 128, 1, 32)])
def test_compact(dt, D, layers, page):
    r = random.Random(D)
    rows, lens = [40, 1, 0, 300, 7, 64], [20, 5, 9, 100, 0, 31]
    b = Batch(dt, 4, 2, D, page, rows, lens)
    k = torch.stack([b.k + i for i in range(layers)])
    v = torch.stack([b.v - i for i in range(layers)])
    path, acc = np.full((6, 301), -1, np.int32), np.array([0, 0, -1, 0, 301, 0], np.int32)
    for s in (0, 3, 5):
        L = {0: 39, 3: 250, 5: 20}[s]
        path[s, :L + 1] = [0] + sorted(r.sample(range(1, rows[s]), L))
        acc[s] = L
    path[1, 0] = 0
    want = [np.stack([ob.compact(f64(t[i]), b.row_start, lens, b.table, path, acc) for i in range(layers)])
            for t in (k, v)]
    ooo.paged_compact(b.batch, k, v, torch.from_numpy(path).cuda(), torch.from_numpy(acc).cuda())
    assert np.array_equal(f64(k), want[0]) and np.array_equal(f64(v), want[1])


def test_compact_leaves_bad_entries():
    b = Batch("bf16", 4, 2, 64, 16, [8, 8], [12, 12])
    b.d_table[1, 1] = -1
    path = torch.tensor([[0, 2, 5, 900], [0, 2, 5, 7]], dtype=torch.int32, device="cuda")
    acc = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    k0 = f64(b.k)
    ooo.paged_compact(b.batch, b.k, b.v, path, acc)
    want = ob.compact(k0, b.row_start, b.lens, b.table, np.array([[0, 2, 5], [0, 2, 5]]), np.array([2, -1]))
    pg, sl = ob.place(b.table[1], 13, 16)  # rows 1 and 3 of sequence 1 lie on its good page; row 4 on does not
    src = ob.place(b.table[1], 14, 16)
    want[pg, :, sl] = k0[src[0], :, src[1]]
    assert np.array_equal(f64(b.k), want)


def test_compact_bounds_rows():
    """Rows past n_rows are none: entries of path that name them stay."""
    b = Batch("bf16", 4, 2, 64, 16, [4, 4], [3, 2])
    b.d_row_start[2] = 1 << 29
    path = torch.tensor([[0, 2, 3, 5], [0, 2, 5, 7]], dtype=torch.int32, device="cuda")
    acc = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    k0 = f64(b.k)
    ooo.paged_compact(b.batch, b.k, b.v, path, acc)
    want = ob.compact(k0, b.row_start, b.lens, b.table, np.array([[0, 2, 3], [0, 2, 2]]), np.array([2, 1]))
    assert np.array_equal(f64(b.k), want)
    b.d_row_start.copy_(torch.tensor([-6, 2, 8], dtype=torch.int32))  # two rows of the first sequence are left
    k0 = f64(b.k)
    ooo.paged_compact(b.batch, b.k, b.v, path, acc * torch.tensor([1, -1], dtype=torch.int32, device="cuda"))
    assert np.array_equal(f64(b.k), k0)  # row 0 stays, 2 and on are none


# ------------------------------------------------------------------ sample


def run_sample(x, T=None, k=None, p=None, m=None, u=None, dt=torch.float32, ld=None):
    n, V = x.shape
    dev = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device="cuda")  # noqa: E731
    f, i = torch.float32, torch.int32
    buf = torch.full((n, ld or V), 1e9, dtype=dt, device="cuda")
    buf[:, :V] = torch.as_tensor(x).to(dt).cuda()
    logits = buf[:, :V]
    ids, kept = (torch.full((n,), -9, dtype=i, device="cuda") for _ in range(2))
    prob = torch.empty(n, device="cuda")
    ws = torch.full((ooo.sample_workspace(n, V),), 0xFF, dtype=torch.uint8, device="cuda")
    u = np.random.default_rng(n * V).random(n).astype(np.float32) if u is None else np.asarray(u, np.float32)
    ooo.sample(logits, dev(u, f), ids, ws, temperature=dev(T, f), top_k=dev(k, i), top_p=dev(p, f), min_p=dev(m, f),
               prob=prob, kept=kept)
    rows = f64(logits)
    f32 = lambda a, r, d: d if a is None else float(np.float32(a[r]))  # noqa: E731
    for r in range(n):
        want = ob.sample(rows[r], f32(T, r, 1.0), 0 if k is None else k[r], f32(p, r, 1.0), f32(m, r, 0.0),
                         float(u[r]))
        got = (int(ids[r]), float(prob[r]), int(kept[r]))
        assert got[0] == want[0] and got[2] == want[2], (r, got, want)
        # one rounding to float32; sums and weights are exact to 2^-42 of the largest, times V
        assert abs(got[1] - want[1]) <= 2 * U32 * want[1] + V * 2.0 ** -42, (r, got, want)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 63, 1000, 1024, 5003, 32000, 151936])
def test_sample_settings(V, dt):
    r = np.random.default_rng(V)
    n = 40 if V <= 5003 else 14
    x = r.normal(0, 2.5, (n, V)).astype(np.float32)
    x[:, r.integers(0, V, 6)] += 6
    x[1:, ::7] = -np.inf if V > 7 else 0
    T = r.choice([0.0, 0.3, 0.7, 1.0, 1.5], n)
    k = r.choice([0, 1, 3, 50, 10 ** 9], n)
    p = r.choice([1.0, 0.999, 0.9, 0.5, 0.0], n)
    m = r.choice([0.0, 0.02, 0.3, 1.0], n)
    run_sample(x, T, k, p, m, dt=dt, ld=V + 3)
    run_sample(x, dt=dt)  # no settings at all
    run_sample(x, T=T, p=p, dt=dt)


@pytest.mark.parametrize("V", [300, 5000, 20011, 140000])
def test_sample_ties(V):
    """Equal logits: all of them, and a few values many times over."""
    r = np.random.default_rng(V)
    x = np.zeros((6, V), np.float32)
    x[1] = -3.25
    x[2] = r.integers(0, 3, V)
    x[3] = np.where(r.random(V) < 0.5, -0.0, 0.0)
    x[4, V // 2:] = 40.0
    x[5] = r.integers(0, 40, V) * 0.5
    for k, p, m in ((0, 1.0, 0.0), (V // 3, 1.0, 0.0), (0, 0.5, 0.0), (V // 2, 0.5, 0.01), (7, 0.3, 0.0)):
        run_sample(x, k=[k] * 6, p=[p] * 6, m=[m] * 6, u=[0.0, 0.25, 0.5, 0.75, 0.999, 0.1])


def test_sample_odd_rows():
    inf, nan = np.inf, np.nan
    x = np.array([[-inf] * 5, [nan] * 5, [nan, 1, -inf, 1, 0], [1, inf, 0, inf, -inf], [-1e38, 1e38, 3e38, -3e38, 0],
                  [-3.4e38] * 5, [0, -inf, nan, nan, -inf]], np.float32)
    for T in (1.0, 0.0, 1e-30, 1e30, float("nan")):
        if T == T:
            run_sample(x, T=[T] * 7, u=[0.6] * 7)
        run_sample(x, T=[1.0] * 7, u=[0.0] * 7)
    run_sample(x, k=[2] * 7, p=[0.99] * 7, u=[0.9999999] * 7)


def test_sample_extreme_settings():
    r = np.random.default_rng(2)
    x = r.normal(0, 3, (8, 3000)).astype(np.float32)
    run_sample(x, T=[0.01, 0.05, 20, 100, 1, 1, 1, 1], k=[0, 0, 0, 0, 2999, 3000, 3001, -4],
               p=[1, .5, .9, 1 - 2.0 ** -24, 1e-30, 2.0, 1 - 2.0 ** -24, 1 - 2.0 ** -24],
               m=[0, 0, 1e-6, 0, 1e-30, -1, 0, 1e-9], u=[1 - 2.0 ** -24] * 8)


@pytest.mark.parametrize("V", [5, 400, 3000, 40000])
def test_sample_counts_above_the_least_floors(V):
    """min_p down to the least float32 over logits far below the largest one:
    tokens of such weights are counted by their logits."""
    r = np.random.default_rng(V)
    x = np.full((7, V), -np.inf, np.float32)
    x[:, :5] = [0, -1, -60, -75, -200]
    x[1:4] = r.uniform(-300, 0, (3, V))
    x[3, V // 2] = np.inf
    x[4] = np.where(np.arange(V) < V - 2, 0.0, -150.0)  # nearly all equal
    x[5] = np.where(np.arange(V) % 3 == 0, np.inf, r.uniform(-300, 0, V))
    x[6] = np.where(np.arange(V) % 2 == 0, -30.0, r.uniform(-100, -30, V))
    for T, m in ((1.0, 1e-30), (0.1, 1e-30), (1.0, 1e-45), (3.0, 1e-18), (1.0, 1e-12))[:5 if V < 40000 else 3]:
        for k in (0, 3, 100, 600):
            run_sample(x, T=[T] * 7, k=[k] * 7, m=[m] * 7, u=[0.0, 0.9, 0.5, 0.3, 0.999, 0.7, 0.1])
        run_sample(x, T=[T] * 7, p=[0.9] * 7, m=[m] * 7, u=[0.0, 0.9, 0.5, 0.3, 0.999, 0.7, 0.1])


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 3000, 40000])
def test_sample_odd_rows_of_every_length(V, dt):
    """Rows of nothing that can be drawn, of infinite logits (more than are
    gathered, too) and of few finite ones, in one workgroup and over many; a
    temperature that is NaN is none."""
    r = np.random.default_rng(V)
    inf, nan = np.inf, np.nan
    x = r.normal(0, 3, (10, V)).astype(np.float32)
    x[0], x[1] = -inf, nan
    x[2] = np.where(r.random(V) < 0.5, nan, -inf)
    x[3, ::5] = nan
    x[3, V // 2] = inf
    x[4, [0, V // 3, V - 1]] = inf
    x[5, ::2] = inf
    x[6] = inf
    x[7] = np.where(r.random(V) < 0.5, nan, -inf)
    x[7, V - 2] = -3.0e38
    x[8] = np.where(r.random(V) < 0.1, nan, np.where(r.random(V) < 0.1, -inf, x[8]))
    x[9] = np.where(r.random(V) < 0.2, inf, np.where(r.random(V) < 0.2, nan, -inf))
    u = [0.0, 0.5, 0.5, 0.9, 0.7, 0.6, 0.9999999, 0.3, 0.8, 0.4]
    for k in (0, 1, 7, 600):
        run_sample(x, k=[k] * 10, u=u, dt=dt)
        run_sample(x, T=[0.7] * 10, k=[k] * 10, p=[0.7] * 10, m=[0.1] * 10, u=u, dt=dt)
    run_sample(x, p=[0.9] * 10, u=u, dt=dt)
    run_sample(x, m=[0.05] * 10, u=u, dt=dt)
    run_sample(x, T=[nan] * 10, k=[7] * 10, p=[0.5] * 10, u=u, dt=dt)
    run_sample(x, T=[0.0, -1.0] * 5, u=u, dt=dt)


@pytest.mark.parametrize("V", [20011, 151936])
@pytest.mark.parametrize("std,T", [(0.3, 1.0), (1.0, 1.0), (0.5, 0.7)])
def test_sample_flat_logits(V, std, T):
    """Different logits so close together that the bins with the places of
    top-p and the draw hold more tokens than are gathered."""
    x = np.random.default_rng(V).normal(0, std, (4, V)).astype(np.float32)
    run_sample(x, T=[T] * 4, p=[0.9, 0.5, 1.0, 0.95], m=[0.0, 0.0, 0.05, 0.2], u=[0.9, 0.3, 0.7, 0.05])


@pytest.mark.parametrize("V", [3000, 70000])
def test_sample_captured_and_replayed(V):
    """Two captured draws with settings of their own on two streams, replayed
    over new logits and numbers: the ids, probabilities and counts of a call."""
    f, i = torch.float32, torch.int32
    sets = [dict(temperature=torch.full((5,), 0.8, device="cuda"), top_k=torch.tensor([0, 1, 40, 600, 0], dtype=i, device="cuda"),
                 top_p=torch.tensor([0.9, 1.0, 0.8, 0.7, 1.0], device="cuda")),
            dict(min_p=torch.full((5,), 0.05, device="cuda"))]
    runs = []
    for kw in sets:
        t = {"x": torch.randn(5, V, device="cuda") * 3, "u": torch.rand(5, device="cuda"),
             "ids": torch.zeros(5, dtype=i, device="cuda"), "prob": torch.zeros(5, dtype=f, device="cuda"),
             "kept": torch.zeros(5, dtype=i, device="cuda"),
             "ws": torch.zeros(ooo.sample_workspace(5, V), dtype=torch.uint8, device="cuda")}
        call = lambda t, kw=kw: ooo.sample(t["x"], t["u"], t["ids"], t["ws"], prob=t["prob"], kept=t["kept"], **kw)  # noqa: E731
        call(t)
        torch.cuda.synchronize()
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call(t)
        runs.append((t, call, s, g))
    for step in range(4):
        for t, *_ in runs:
            t["x"].normal_(0, 3 - 0.7 * step)
            t["u"].uniform_()
            t["ws"].fill_(0xFF)
        torch.cuda.synchronize()
        for _, _, s, g in runs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for t, call, *_ in runs:
            got = [t[n].clone() for n in ("ids", "prob", "kept")]
            call(t)
            assert all(torch.equal(a, t[n]) for a, n in zip(got, ("ids", "prob", "kept")))
            assert (t["ids"] >= 0).all()


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_steps_captured_and_replayed(dt):
    """Append, plan, attention, compaction and a draw as one captured step,
    replayed while lengths and tables grow, each replay against the reference
    and against the same calls made one by one."""
    r = random.Random(11)
    rows, lens = [4, 1, 6, 3], [30, 14, 0, 77]
    mask = bh.trie_masks(r, rows, 1)[0]
    depth = np.array([bin(int(m[0])).count("1") - 1 for m in mask], np.int32)
    Hq, Hkv, D, page, shared = 8, 2, 64, 16, 45
    room = [n + 40 for n in lens]  # page tables with room for five steps
    a, e = (Batch(dt, Hq, Hkv, D, page, rows, room, shared=shared, mask=mask, seed=3, table_pad=0) for _ in range(2))
    width, V = (Hq + 2 * Hkv) * D, 500
    bufs = []
    for b in (a, e):
        b.lens = list(lens)
        b.d_len.copy_(torch.tensor(lens, dtype=torch.int32))
        t = {"qkv": torch.zeros(b.n_rows, width, dtype=b.dt, device="cuda"), "q": torch.zeros_like(b.q),
             "out": torch.zeros_like(b.q), "depth": torch.from_numpy(depth).cuda(),
             "path": torch.full((4, 7), -1, dtype=torch.int32, device="cuda"),
             "acc": torch.zeros(4, dtype=torch.int32, device="cuda"), "u": torch.zeros(b.n_rows, device="cuda"),
             "ids": torch.zeros(b.n_rows, dtype=torch.int32, device="cuda"),
             "logits": torch.zeros(b.n_rows, V, device="cuda"),
             "plan": torch.zeros(ooo.paged_plan_bytes(b.batch), dtype=torch.uint8, device="cuda"),
             "ws": torch.zeros(ooo.paged_attn_workspace(b.batch), dtype=torch.uint8, device="cuda"),
             "sws": torch.zeros(ooo.sample_workspace(b.n_rows, V), dtype=torch.uint8, device="cuda")}
        t["k2"], t["v2"] = b.k[None], b.v[None]
        bufs.append(t)
    w = torch.randn(Hq * D, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") / 8

    def attend(b, t):
        ooo.paged_append(b.batch, t["qkv"], None, None, 1e-6, 1e6, t["q"], b.k, b.v, depth=t["depth"])
        ooo.paged_plan(b.batch, t["plan"])
        ooo.paged_attn(b.batch, t["plan"], t["q"], b.k, b.v, b.scale, t["out"], t["ws"])

    def finish(b, t):
        ooo.sample(t["logits"], t["u"], t["ids"], t["sws"])
        ooo.paged_compact(b.batch, t["k2"], t["v2"], t["path"], t["acc"])
        b.d_len.add_(t["acc"] + 1)

    stream = torch.cuda.Stream()
    graphs = []
    attend(a, bufs[0])  # everything is loaded before the capture
    finish(a, bufs[0])
    a.d_len.copy_(torch.tensor(lens, dtype=torch.int32))
    a.k.copy_(e.k)
    a.v.copy_(e.v)
    torch.cuda.synchronize()
    for f in (attend, finish):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            f(a, bufs[0])
        graphs.append(g)
    for step in range(5):
        gen = torch.Generator(device="cuda").manual_seed(100 + step)
        qkv = torch.randn(a.n_rows, width, generator=gen, device="cuda").to(a.dt)
        u = torch.rand(a.n_rows, generator=gen, device="cuda")
        path, acc = np.full((4, 7), -1, np.int32), np.zeros(4, np.int32)
        for s, n in enumerate(rows):
            node = r.randrange(n)  # the path from the root to a random node
            p = [j for j in range(n) if (int(mask[a.row_start[s] + node, 0]) >> j) & 1]
            path[s, :len(p)], acc[s] = p, len(p) - 1
        for t in bufs:
            t["qkv"].copy_(qkv)
            t["u"].copy_(u)
            t["path"].copy_(torch.from_numpy(path))
            t["acc"].copy_(torch.from_numpy(acc))
        torch.cuda.synchronize()
        graphs[0].replay()
        attend(e, bufs[1])
        torch.cuda.synchronize()
        assert torch.equal(bufs[0]["out"], bufs[1]["out"])
        a.q = bufs[0]["q"]
        a.check(bufs[0]["out"])
        for t in bufs:
            t["logits"].copy_(t["out"].float().view(a.n_rows, -1) @ w)
        want_k = ob.compact(f64(a.k), a.row_start, a.lens, a.table, path, acc)
        torch.cuda.synchronize()
        graphs[1].replay()
        finish(e, bufs[1])
        torch.cuda.synchronize()
        assert torch.equal(bufs[0]["ids"], bufs[1]["ids"]) and torch.equal(a.k, e.k) and torch.equal(a.v, e.v)
        assert np.array_equal(f64(a.k), want_k)
        x = f64(bufs[0]["logits"])
        for row in range(a.total):
            assert int(bufs[0]["ids"][row]) == ob.sample(x[row], 1.0, 0, 1.0, 0.0, float(u[row]))[0]
        for b in (a, e):
            b.lens = [n + int(c) + 1 for n, c in zip(b.lens, acc)]
        assert a.d_len.tolist() == a.lens


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_layers_interleaved_in_one_pool(dt):
    """Pages that hold the rows of three layers: one layer's calls and a
    compaction of all of them leave the others' rows alone."""
    r = random.Random(8)
    rows, lens = [20, 3, 9], [25, 60, 7]
    mask, depth = bh.trie_masks(r, rows, 1)
    b = Batch(dt, 4, 2, 64, 16, rows, lens, shared=21, mask=mask, seed=6)
    n, Hkv, R, D = b.k.shape
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((n, 3, Hkv, R, D), generator=g, device="cuda").to(b.dt).transpose(0, 1) for _ in range(2))
    b.k, b.v = k[1], v[1]
    b.batch = ooo.PagedBatch(b.d_row_start, b.d_len, b.d_table, b.k, 4, b.n_rows, shared_pages=b.d_shared,
                             shared_len=21, anc_mask=b.d_mask)
    others = [f64(t[i]) for t in (k, v) for i in (0, 2)]
    run_append(b, True, depth)
    b.check(b.attend())
    assert all(np.array_equal(a, f64(t)) for a, t in zip(others, [t[i] for t in (k, v) for i in (0, 2)]))
    path, acc = np.full((3, 20), -1, np.int32), np.array([4, -1, 2], np.int32)
    path[0, :5], path[2, :3] = [0, 3, 8, 9, 19], [0, 1, 7]
    want = [np.stack([ob.compact(f64(t[i]), b.row_start, lens, b.table, path, acc) for i in range(3)]) for t in (k, v)]
    ooo.paged_compact(b.batch, k, v, torch.from_numpy(path).cuda(), torch.from_numpy(acc).cuda())
    assert np.array_equal(f64(k), want[0]) and np.array_equal(f64(v), want[1])
