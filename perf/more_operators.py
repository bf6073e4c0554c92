"""The operators of a batched step over an 8-bit cache that are measured, with
their plain forms.

A batch of requests shares one long tool prompt and keeps keys and values in
cache pages of e4m3 numbers, with one power of two for each block of 32 tokens
and KV head (K and V apart): appending rows (head norms, rotation, quantisation
and, where a later token needs it, a larger scale for the block's earlier rows:
``append8``), attention over the shared prompt and each sequence's own pages
(``attn8``), moving the accepted rows of a batch of tries together, between
blocks of different scales (``compact8``), and continuing one request several
times from its cache (``fork``: whole pages are shared, the open one is copied;
for caches of 8, 16 and 32 bits).

Sizes are the repository's workload shapes (``workload.py``: 32 query and 8
KV heads of 128, 16 and 8, 40 and 8, one KV head of 64 in float32; prompts of
128 to 32768 rows; tries of 25 to 256 nodes) and generic ones.  A case's
``mix`` fixes its ragged lengths and tries; the values come from the seed.
"""

import math
import random

import numpy as np
import torch

own = False

EPS = 1.0e-6
THETA = 1.0e6
BLOCK = 32             # tokens of a scale
LOW, HIGH = -100, 119  # exponents of a scale
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f8": torch.float8_e4m3fn}


def listed():
    return [
        # A float32 trie step of one small request: latency of the smallest append.
        {"name": "append8_f32_trie", "kind": "append8", "dt": "f32", "Hq": 4, "Hkv": 1, "D": 64, "seqs": 1, "rows": 25,
         "ragged": False, "trie": True, "shared": 128, "own": 64, "page": 32, "norm": True, "pad": 0, "mix": 1},
        # The next token of 256 requests: an ordinary decoding step, each row in a block of its own.
        {"name": "append8_decode_256", "kind": "append8", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 256,
         "rows": 1, "ragged": False, "trie": False, "shared": 4096, "own": 512, "page": 64, "norm": True, "pad": 0,
         "mix": 2},
        # Prompts of 16 requests coming in at once, ragged, behind a common prefix: the bandwidth of an append.
        {"name": "append8_prompts", "kind": "append8", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 16,
         "rows": 1024, "ragged": True, "trie": False, "shared": 4096, "own": 512, "page": 64, "norm": True, "pad": 37,
         "mix": 3},
        # Float32 tries of three requests over a short prompt: the float32 option, small.
        {"name": "attn8_f32_tries", "kind": "attn8", "dt": "f32", "Hq": 4, "Hkv": 1, "D": 64, "seqs": 3, "rows": 25,
         "ragged": True, "trie": True, "shared": 128, "own": 100, "page": 32, "pad": 0, "mix": 4},
        # Plain decoding of 64 requests over a 4k tool prompt: the ordinary serving step.
        {"name": "attn8_decode_64", "kind": "attn8", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 64, "rows": 1,
         "ragged": False, "trie": False, "shared": 4096, "own": 2048, "page": 64, "pad": 0, "mix": 5},
        # Eight requests verifying tries of up to 64 nodes over the same prompt: the batched verify step.
        {"name": "attn8_tries_8", "kind": "attn8", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 8, "rows": 64,
         "ragged": True, "trie": True, "shared": 4096, "own": 512, "page": 32, "pad": 5, "mix": 6},
        # Chunks of four requests' own prompts, up to 512 rows each, behind a 1k prompt (Qwen3-0.6B heads).
        {"name": "attn8_prompts_4", "kind": "attn8", "dt": "bf16", "Hq": 16, "Hkv": 8, "D": 128, "seqs": 4,
         "rows": 512, "ragged": True, "trie": False, "shared": 1024, "own": 300, "page": 128, "pad": 0, "mix": 7},
        # 256 requests late in their calls over a 32k prompt: the largest step, twice as long as 16 bits would hold.
        {"name": "attn8_decode_256", "kind": "attn8", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 256,
         "rows": 1, "ragged": False, "trie": False, "shared": 32768, "own": 4096, "page": 32, "pad": 0, "mix": 8},
        # One request's accepted rows, one layer: the smallest commit.
        {"name": "compact8_one", "kind": "compact8", "dt": "f32", "Hkv": 1, "D": 64, "layers": 1, "seqs": 1,
         "rows": 25, "own": 100, "page": 32, "mix": 9},
        # The commit of eight requests over all 36 layers.
        {"name": "compact8_36x8", "kind": "compact8", "dt": "bf16", "Hkv": 8, "D": 128, "layers": 36, "seqs": 8,
         "rows": 64, "own": 512, "page": 32, "mix": 10},
        # A second try of one small float32 request, one layer: the smallest fork.
        {"name": "fork_f32_one", "kind": "fork", "dt": "f32", "Hkv": 1, "D": 64, "layers": 1, "seqs": 1, "children": 1,
         "own": 100, "page": 16, "mix": 11},
        # Eight samples each of eight requests, all 36 layers of an 8-bit cache.
        {"name": "fork_f8_36x64", "kind": "fork", "dt": "f8", "Hkv": 8, "D": 128, "layers": 36, "seqs": 8,
         "children": 64, "own": 1024, "page": 64, "mix": 12},
    ]


# ---------------------------------------------------------------- drawing


def _log(rng, lo, hi):
    """An integer between lo and hi, its logarithm spread evenly."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append8"] * 3 + ["attn8"] * 5 + ["compact8"] * 2 + ["fork"] * 2)
    mix = rng.randrange(1 << 30)
    D = rng.choice([64, 128, 128])
    page = rng.choice([32, 64, 128])
    if kind == "fork":
        dt = rng.choice(["f8", "f8", "bf16", "f32"])
        seqs = _log(rng, 1, 16)
        return {"kind": kind, "dt": dt, "Hkv": rng.choice([1, 2, 4, 8]), "D": D, "layers": _log(rng, 1, 36),
                "seqs": seqs, "children": _log(rng, 1, 64), "own": _log(rng, 1, 1024),
                "page": page if dt == "f8" else rng.choice([16, 32, 64, 128]), "mix": mix}
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "compact8":
        return {"kind": kind, "dt": dt, "Hkv": rng.choice([1, 2, 4, 8]), "D": D, "layers": _log(rng, 1, 36),
                "seqs": _log(rng, 1, 8), "rows": _log(rng, 2, 64), "own": _log(rng, 1, 512), "page": page, "mix": mix}
    Hq, Hkv = rng.choice([(4, 1), (8, 8), (14, 2), (16, 8), (32, 8), (32, 8), (40, 8)])
    trie = rng.random() < 0.4
    common = {"kind": kind, "dt": dt, "Hq": Hq, "Hkv": Hkv, "D": D, "ragged": rng.random() < 0.7, "trie": trie}
    if kind == "append8":
        rows = rng.choice([1, _log(rng, 1, 256 if trie else 1024)])
        return {**common, "seqs": _log(rng, 1, max(1, min(256, 16384 // rows))), "rows": rows,
                "shared": _log(rng, 1, 32768), "own": _log(rng, 1, 2048), "page": page, "norm": rng.random() < 0.7,
                "pad": rng.choice([0, 0, 3, 50]), "mix": mix}
    rows = rng.choice([1, 1, _log(rng, 2, 256), _log(rng, 2, 256 if trie else 512)])
    seqs = _log(rng, 1, max(1, min(256, 2048 // rows)))
    shared = rng.choice([0, _log(rng, 16, 32768), _log(rng, 16, 32768)])
    own_len = _log(rng, 1, 4096)
    while 4 * Hq * D * seqs * rows * (shared + own_len + rows) > (1.4e11 if dt == "bf16" else 4e10):
        shared, own_len = shared // 2, max(1, own_len // 2)
    return {**common, "seqs": seqs, "rows": rows, "shared": shared, "own": own_len, "page": page,
            "pad": rng.choice([0, 0, 3, 50]), "mix": mix}


# ----------------------------------------------------------------- inputs


def _lengths(case):
    """New rows and own committed rows of every sequence, from the case alone."""
    r = random.Random(case["mix"])
    rows, lens = [], []
    for _ in range(case["seqs"]):
        n = case.get("rows", 0)
        rows.append(r.randint(max(1, n // 4), n) if case.get("ragged") else n)
        lens.append(r.randint(case["own"] // 8, case["own"]))
    return rows, lens


def _forks(case):
    """Which sequence each child of a fork case continues."""
    r = random.Random(case["mix"] + 3)
    return [r.randrange(case["seqs"]) for _ in range(case["children"])]


def _parents(r, n):
    """A trie as drafts make it: long runs with a few branches."""
    return [-1] + [i - 1 if r.random() < 0.85 else r.randrange(i) for i in range(1, n)]


def _tries(case, rows):
    """Depths [rows] and ancestor masks [rows][words] of the batch's tries."""
    r = random.Random(case["mix"] + 1)
    words = max(1, (max(rows) + 63) // 64)
    depth, masks = [], []
    for n in rows:
        m = np.zeros((n, words), np.uint64)
        d = []
        for i, p in enumerate(_parents(r, n)):
            if p >= 0:
                m[i] = m[p]
            d.append(0 if p < 0 else d[p] + 1)
            m[i, i >> 6] |= np.uint64(1) << np.uint64(i & 63)
        depth += d
        masks.append(m)
    return np.array(depth, np.int32), np.concatenate(masks).view(np.int64)


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _randn(shape, seed, stream, dtype, std=1.0, mean=0.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat, g, step = out.view(-1), _gen(seed, stream), 1 << 27
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device="cuda").mul_(std).add_(mean)
    return out


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _exponent(amax):
    """The least e with amax <= 448 2^e, bounded (float32 in, whole numbers out)."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(amax > 0, e, LOW).clamp(LOW, HIGH).int()


def _cache(lead, n_pages, Hkv, R, D, seed, stream):
    """A pool of 8-bit pages and its scales, of tokens whose size varies as keys' and values' do."""
    shape = (*lead, n_pages, Hkv, R, D)
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((*lead, n_pages, Hkv, R // BLOCK), dtype=torch.uint8, device="cuda")
    c, s, g = codes.view(-1, BLOCK, D), scales.view(-1), _gen(seed, stream)
    step = (1 << 27) // (BLOCK * D)
    for i in range(0, c.shape[0], step):
        n = min(step, c.shape[0] - i)
        x = torch.randn((n, BLOCK, D), generator=g, device="cuda")
        x *= torch.randn((n, BLOCK, 1), generator=g, device="cuda").mul_(0.4).exp_()
        e = _exponent(x.abs().amax((1, 2)))
        c[i:i + n] = _codes(x, e[:, None, None])
        s[i:i + n] = (e + 127).to(torch.uint8)
    return codes, scales.view(torch.float8_e8m0fnu)


def _batch(case, seed):
    """Page tables and lengths of a batch; the pool's pages are handed out in random order, two of them unused."""
    rows, lens = _lengths(case)
    R = case["page"]
    need = [(n + m + R - 1) // R for n, m in zip(rows, lens)]
    need = [max(n, m // R + 1) for n, m in zip(need, lens)] if case["kind"] == "fork" else need
    ns = (case.get("shared", 0) + R - 1) // R
    children = case.get("children", 0)
    n_pages = sum(need) + ns + children + 2
    ids = np.random.default_rng(int(seed) % (1 << 32)).permutation(n_pages).astype(np.int32)
    table = np.zeros((len(rows) + children, max(need) + (1 if children else 0)), np.int32)
    at = ns
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    total = sum(rows)
    return {"rows": rows, "lens": lens, "total": total, "n_rows": max(1, total + case.get("pad", 0)),
            "n_pages": n_pages, "row_start": _dev(np.cumsum([0] + rows + [0] * children).astype(np.int32)),
            "seq_len": _dev(np.array(lens + [0] * children, np.int32)), "table": _dev(table),
            "fresh": _dev(np.concatenate([np.full(len(rows), -1, np.int32), ids[at:at + children]])),
            "shared_pages": _dev(ids[:ns]) if ns else None}


def prepare(case, seed):
    kind = case["kind"]
    st = {"case": case}
    b = _batch(case, seed)
    st.update(b)
    R, Hkv, D = case["page"], case["Hkv"], case["D"]
    lead = (case["layers"],) if kind in ("compact8", "fork") else ()
    if case["dt"] == "f8" or kind != "fork":
        st["k"], st["ks"] = _cache(lead, b["n_pages"], Hkv, R, D, seed, 1)
        st["v"], st["vs"] = _cache(lead, b["n_pages"], Hkv, R, D, seed, 2)
    else:
        shape = (*lead, b["n_pages"], Hkv, R, D)
        st["k"], st["v"] = _randn(shape, seed, 1, TYPES[case["dt"]]), _randn(shape, seed, 2, TYPES[case["dt"]])
    n = b["n_rows"]
    if kind == "compact8":
        r = random.Random(case["mix"] + 2 + seed)
        cap = max(b["rows"]) + 1
        path, acc = np.full((case["seqs"], cap), -1, np.int32), np.zeros(case["seqs"], np.int32)
        for s, m in enumerate(b["rows"]):  # a root path of the sequence's trie
            L = r.randint(0, m - 1)
            path[s, :L + 1] = [0] + sorted(r.sample(range(1, m), L))
            acc[s] = L
        st["path"], st["accept"] = _dev(path), _dev(acc)
    elif kind == "fork":
        st["parent"] = _dev(np.array([-1] * case["seqs"] + _forks(case), np.int32))
    else:
        Hq, dt = case["Hq"], TYPES[case["dt"]]
        st["mask"] = st["depth"] = None
        if case["trie"]:
            depth, mask = _tries(case, b["rows"])
            pad = n - b["total"]
            st["depth"] = _dev(np.concatenate([depth, np.zeros(pad, np.int32)]))
            st["mask"] = _dev(np.concatenate([mask, np.zeros((pad, mask.shape[1]), np.int64)]))
        if kind == "append8":
            x = _randn((n, (Hq + 2 * Hkv) * D), seed, 3, torch.float32)
            st["qkv"] = (x * _randn((n, 1), seed, 7, torch.float32, 0.4).exp_()).to(dt)
            norm = case["norm"]
            st["qw"] = _randn((D,), seed, 4, dt, 0.1, 1.0) if norm else None
            st["kw"] = _randn((D,), seed, 5, dt, 0.1, 1.0) if norm else None
            st["q_out"] = _randn((n, Hq, D), seed, 6, dt)
        else:
            st["q"] = _randn((n, Hq, D), seed, 3, dt)
            st["out"] = _randn((n, Hq, D), seed, 6, dt, 0.02)
            st["scale"] = 1.0 / math.sqrt(D)
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    """What a serving program keeps: the batch's descriptor, the cache's, the step's plan (one for all its layers) and scratch."""
    from paper_2608_00814_amd import ooo

    case = st["case"]
    pages = st["k"][0] if st["k"].dim() == 5 else st["k"]
    eight = pages.dtype == torch.float8_e4m3fn
    more = {"dtype": torch.bfloat16 if case["kind"] == "fork" else TYPES[case["dt"]]} if eight else {}
    st["batch"] = ooo.PagedBatch(st["row_start"], st["seq_len"], st["table"], pages, case.get("Hq", case["Hkv"]),
                                 n_rows=st["n_rows"], shared_pages=st["shared_pages"],
                                 shared_len=case.get("shared", 0), anc_mask=st.get("mask"), **more)
    if eight:
        st["cache"] = ooo.Cache8(st["batch"], st["k"], st["v"], st["ks"], st["vs"])
    if case["kind"] == "attn8":
        st["plan"] = ooo.paged_plan8(st["batch"])
        st["ws"] = torch.empty(ooo.paged_attn8_workspace(st["batch"]), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------- runs


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own[kind](state)
    return _plain[kind](state)


def _own_append8(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_append8(s["batch"], s["cache"], s["qkv"], s["qw"], s["kw"], EPS, THETA, s["q_out"], depth=s["depth"])
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _own_attn8(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_attn8(s["batch"], s["cache"], s["plan"], s["q"], s["scale"], s["out"], s["ws"])
    return s["out"]


def _own_compact8(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_compact8(s["batch"], s["cache"], s["path"], s["accept"])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _own_fork(s):
    from paper_2608_00814_amd import ooo

    if "cache" in s:
        ooo.paged_fork8(s["batch"], s["cache"], s["parent"], s["fresh"], s["seq_len"], s["table"])
    else:
        ooo.paged_fork(s["batch"], s["k"], s["v"], s["parent"], s["fresh"], s["seq_len"], s["table"])
    return _forked(s)


def _forked(s):
    out = {"seq_len": s["seq_len"], "table": s["table"], "k": s["k"], "v": s["v"]}
    return {**out, "ks": s["ks"], "vs": s["vs"]} if "ks" in s else out


_own = {"append8": _own_append8, "attn8": _own_attn8, "compact8": _own_compact8, "fork": _own_fork}


def _rows_of(s):
    """Sequence and index in it of every row (rows behind the last sequence: those of row 0), and which are real."""
    r = torch.arange(s["n_rows"], device="cuda")
    real = r < s["row_start"][-1]
    r = torch.where(real, r, 0)
    b = torch.searchsorted(s["row_start"][1:].contiguous(), r.int(), right=True)
    return b, r - s["row_start"][b], real, r


def _codes(x, e):
    """x / 2^e as e4m3 numbers (the power from its bits: a rounded one would move ties)."""
    down = (1023 - e.long() << 52).view(torch.float64).float()
    return (x * down).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_append8(s):
    c = s["case"]
    Hq, Hkv, D, R = c["Hq"], c["Hkv"], c["D"], c["page"]
    b, i, real, r = _rows_of(s)
    x = s["qkv"][r].float().view(-1, Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if c["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["qw"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["kw"].float()
    slot = s["seq_len"][b] + i
    depth = i if s["depth"] is None else s["depth"][r]
    j = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    ang = (c["shared"] + s["seq_len"][b] + depth).double()[:, None] * THETA ** (-2.0 * j / D)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def turned(t):
        lo, hi = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

    s["q_out"].copy_(torch.where(real[:, None, None], turned(q).to(s["qkv"].dtype), s["q_out"]))
    # blocks of the pool, by page and place in it
    B, n_blocks = R // BLOCK, s["n_pages"] * (R // BLOCK)
    page = s["table"][b, slot // R].long()
    block = page * B + slot % R // BLOCK
    first = s["seq_len"] // BLOCK * BLOCK                      # where each sequence's open block begins, if there is one
    more = s["row_start"][1:] > s["row_start"][:-1]
    open_ = (s["seq_len"] > first) & more
    opage = s["table"].gather(1, (first // R)[:, None].long())[:, 0].long()
    oblock = torch.where(open_, opage * B + first % R // BLOCK, n_blocks)
    orow = first[:, None] % R + torch.arange(BLOCK, device="cuda")
    held = (torch.arange(BLOCK, device="cuda") < (s["seq_len"] - first)[:, None]) & more[:, None]
    for pool, scales, t in ((s["k"], s["ks"], turned(k)), (s["v"], s["vs"], v)):
        codes, bytes_ = pool.view(torch.uint8), scales.view(torch.uint8)
        old = bytes_.permute(0, 2, 1).reshape(n_blocks, Hkv).int() - 127
        amax = torch.zeros((n_blocks, Hkv), device="cuda").index_reduce_(0, block, t.abs().amax(-1), "amax")
        touched = torch.zeros(n_blocks + 1, dtype=torch.bool, device="cuda")
        touched[block] = True
        kept = torch.zeros(n_blocks + 1, dtype=torch.bool, device="cuda")
        kept[oblock] = True
        need = _exponent(amax)
        new = torch.where(kept[:-1, None], torch.maximum(old, need), need)
        new = torch.where(touched[:-1, None], new, old)
        # the rows that the open blocks hold, under the scales that these get
        o = oblock.clamp(max=n_blocks - 1)
        was = codes[opage[:, None], :, orow].view(torch.float8_e4m3fn)           # [sequences][BLOCK][Hkv][D]
        now = _codes(was.float(), (new[o] - old[o])[:, None, :, None])
        codes[opage[:, None], :, orow] = torch.where(held[:, :, None, None] & open_[:, None, None, None],
                                                     now.view(torch.uint8), was.view(torch.uint8))
        codes[page, :, slot % R] = _codes(t, new[block][..., None]).view(torch.uint8)
        bytes_.copy_((new + 127).to(torch.uint8).view(-1, B, Hkv).permute(0, 2, 1))
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _values(codes, scales):
    """What pages [..., R, D] with scales [..., R / BLOCK] stand for, in float32."""
    x = codes.float().unflatten(-2, (-1, BLOCK))
    return (x * scales.float()[..., None, None]).flatten(-3, -2)


def _plain_attn8(s):
    c = s["case"]
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["shared"]
    G, B, most = Hq // Hkv, c["seqs"], max(s["rows"])
    start, lens = s["row_start"][:-1].long(), s["seq_len"].long()
    count = s["row_start"][1:].long() - start
    i = torch.arange(most, device="cuda")
    at = torch.where(i < count[:, None], start[:, None] + i, 0)                     # [B][most]
    q = s["q"][at].float().view(B, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * G, D)
    pools = ((s["k"].view(torch.uint8), s["ks"].view(torch.uint8)), (s["v"].view(torch.uint8), s["vs"].view(torch.uint8)))

    def values(pages, pool):  # pages [...] -> [..., Hkv, R, D]
        codes, scales = pool
        return _values(codes[pages].view(torch.float8_e4m3fn), scales[pages].view(torch.float8_e8m0fnu))

    kv = [values(s["table"].long(), p).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D) for p in pools]
    key = torch.arange(kv[0].shape[2], device="cuda")
    new = key - lens[:, None]                                                       # [B][keys]: index among the new rows
    if s["mask"] is None:
        ok = new[:, None] <= i[:, None]
    else:
        words = s["mask"][at]                                                       # [B][most][words]
        n = new.clamp(0, 64 * words.shape[2] - 1)[:, None].expand(B, most, -1)
        bit = (torch.gather(words, 2, n >> 6) >> (n & 63)) & 1
        ok = (new[:, None] < 0) | ((bit == 1) & (new < count[:, None])[:, None])
    x = torch.matmul(q, kv[0].transpose(-1, -2)).view(B, Hkv, most, G, -1) * s["scale"]
    x = x.masked_fill_(~ok[:, None, :, None], float("-inf")).view(B, Hkv, most * G, -1)
    top = x.amax(-1, keepdim=True)
    if S:
        shared = [values(s["shared_pages"].long(), p).transpose(0, 1).reshape(Hkv, -1, D)[:, :S] for p in pools]
        y = torch.matmul(q, shared[0].transpose(-1, -2)) * s["scale"]
        top = torch.maximum(top, y.amax(-1, keepdim=True))
    x = x.sub_(top).exp_()
    den = x.sum(-1, keepdim=True)
    o = torch.matmul(x, kv[1])
    if S:
        y = y.sub_(top).exp_()
        den = den + y.sum(-1, keepdim=True)
        o = o + torch.matmul(y, shared[1])
    o = (o / den).view(B, Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(B, most, Hq, D)
    b, i, real, _ = _rows_of(s)
    s["out"].copy_(torch.where(real[:, None, None], o[b, i].to(s["out"].dtype), s["out"]))
    return s["out"]


def _plain_compact8(s):
    R, Hkv = s["case"]["page"], s["case"]["Hkv"]
    B, n_blocks = R // BLOCK, s["n_pages"] * (R // BLOCK)
    d = torch.arange(s["path"].shape[1], device="cuda")
    on = d <= s["accept"][:, None]
    base = s["seq_len"][:, None]
    src = base + torch.where(on, s["path"], 0)
    dst = base + torch.where(on, d, 0)  # entries behind the path move the root to itself
    b = torch.arange(on.shape[0], device="cuda")[:, None].expand_as(src)
    sp, dp = s["table"][b, src // R].long(), s["table"][b, dst // R].long()
    from_, to = sp * B + src % R // BLOCK, dp * B + dst % R // BLOCK
    first = s["seq_len"] // BLOCK * BLOCK
    opage = s["table"].gather(1, (first // R)[:, None].long())[:, 0].long()
    oblock = opage * B + first % R // BLOCK
    held = torch.arange(BLOCK, device="cuda") < (s["seq_len"] - first)[:, None]
    orow = first[:, None] % R + torch.arange(BLOCK, device="cuda")
    for pool, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        L = pool.shape[0]
        codes, bytes_ = pool.view(torch.uint8), scales.view(torch.uint8)
        old = bytes_.permute(1, 3, 0, 2).reshape(n_blocks, L, Hkv).int() - 127
        e = old[from_]                                                            # [sequences][path][L][Hkv]
        new = torch.full((n_blocks, L, Hkv), -1000, dtype=torch.int32, device="cuda")
        new.view(n_blocks, -1).index_reduce_(0, to.reshape(-1), e.reshape(-1, L * Hkv), "amax")
        touched = new > -1000
        has = torch.zeros(n_blocks, dtype=torch.bool, device="cuda")
        has[oblock] = s["seq_len"] > first
        new = torch.where(has[:, None, None], torch.maximum(new, old), new)
        new = torch.where(touched, new, old)
        x = codes[:, sp, :, src % R].view(torch.float8_e4m3fn).float()            # [sequences][path][L][Hkv][D]
        x = _codes(x, (new[to] - e)[..., None]).view(torch.uint8)
        was = codes[:, opage[:, None], :, orow].view(torch.float8_e4m3fn)         # [sequences][BLOCK][L][Hkv][D]
        now = _codes(was.float(), (new[oblock] - old[oblock])[:, None, :, :, None])
        codes[:, opage[:, None], :, orow] = torch.where(held[:, :, None, None, None], now.view(torch.uint8),
                                                        was.view(torch.uint8))
        codes[:, dp, :, dst % R] = x
        bytes_.copy_((new + 127).to(torch.uint8).view(-1, B, L, Hkv).permute(2, 0, 3, 1))
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _plain_fork(s):
    R = s["case"]["page"]
    p = s["parent"]
    b = torch.nonzero(p >= 0)[:, 0]
    p = p[b].long()
    n, at = s["seq_len"][p], s["seq_len"][p] // R
    src, dst = s["table"][p, at.long()].long(), s["fresh"][b].long()
    rows = torch.arange(R, device="cuda") < (n % R)[:, None]                        # [children][R]
    parts = [(s["k"], rows[..., None]), (s["v"], rows[..., None])]
    if "ks" in s:
        parts += [(s["ks"], rows[:, ::BLOCK]), (s["vs"], rows[:, ::BLOCK])]
    for pool, here in parts:
        t = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        t[:, dst] = torch.where(here[:, None], t[:, src], t[:, dst])
    entry = torch.arange(s["table"].shape[1], device="cuda")
    row = torch.where(entry < at[:, None], s["table"][p], s["table"][b])
    s["table"][b] = torch.where(entry == at[:, None], s["fresh"][b][:, None], row)
    s["seq_len"][b] = n
    return _forked(s)


_plain = {"append8": _plain_append8, "attn8": _plain_attn8, "compact8": _plain_compact8, "fork": _plain_fork}


# ------------------------------------------------------------------- work


def work(case):
    kind, e = case["kind"], {"f32": 4, "bf16": 2, "f8": 1}[case["dt"]]
    rows, lens = _lengths(case)
    total, D, Hkv = sum(rows), case["D"], case["Hkv"]
    if kind == "compact8":
        return {"bytes": 4.0 * case["layers"] * total / 2 * Hkv * D, "flops": 0}
    if kind == "fork":
        moved = sum(lens[p] % case["page"] for p in _forks(case))
        return {"bytes": 4.0 * case["layers"] * moved * Hkv * D * e + 64.0 * case["children"], "flops": 0}
    Hq = case["Hq"]
    if kind == "append8":
        return {"bytes": float(total) * D * (e * (2 * Hq + 2 * Hkv) + 2 * Hkv),
                "flops": 8.0 * total * (Hq + 2 * Hkv) * D}
    own_keys = sum(rows) + sum(lens)
    if case["trie"]:
        r = random.Random(case["mix"] + 1)
        seen = 0
        for n, m in zip(rows, lens):
            d = []
            for p in _parents(r, n):
                d.append(0 if p < 0 else d[p] + 1)
            seen += n * m + sum(d) + n
    else:
        seen = sum(n * m + n * (n + 1) // 2 for n, m in zip(rows, lens))
    return {"bytes": float(e) * 2 * total * Hq * D + 2.0 * Hkv * D * (case["shared"] + own_keys),
            "flops": 4.0 * Hq * D * (seen + total * case["shared"])}


# ------------------------------------------------------------------ exact


def exact(case, seed):
    """The definitions in 64 bits, one sequence after the other."""
    if case["kind"] == "fork":
        return None  # rows are moved, nothing is computed
    s = prepare(case, seed)
    return {"append8": _exact_append8, "attn8": _exact_attn8, "compact8": _exact_compact8}[case["kind"]](case, s)


def _e4m3(y):
    """y (64 bits, |y| <= 448) to three bits behind the leading one, ties to even, none below 2^-9."""
    _, e = torch.frexp(y)
    step = _two((e - 1).clamp_min(-6) - 3)
    return torch.round(y / step) * step


def _two(e):
    """2^e in 64 bits for whole e."""
    table = torch.tensor([math.ldexp(1.0, k) for k in range(-600, 601)], dtype=torch.float64, device=e.device)
    return table[e.long() + 600]


def _least(amax):
    """The least whole e with amax <= 448 2^e, within its bounds, for every element."""
    e = torch.ceil(torch.log2(amax / 448.0)).clamp(LOW, HIGH)  # to be put right by one where the logarithm was rounded
    e = torch.where(amax > 448.0 * _two(e), e + 1, e)
    e = torch.where(amax <= 448.0 * _two(e - 1), e - 1, e)
    return e.clamp(LOW, HIGH)


def _exact_append8(c, s):
    Hq, Hkv, D, R = c["Hq"], c["Hkv"], c["D"], c["page"]
    q_out = s["q_out"].double()
    pools = {n: s[n].double() for n in ("k", "v", "ks", "vs")}
    depth = None if s["depth"] is None else s["depth"].tolist()
    table = s["table"].tolist()
    first = 0
    freq = torch.tensor([math.pow(THETA, -2.0 * j / D) for j in range(D // 2)], dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(zip(s["rows"], s["lens"])):
        x = s["qkv"][first:first + n].double().reshape(n, Hq + 2 * Hkv, D)
        steps = list(range(n)) if depth is None else depth[first:first + n]
        a = torch.tensor([c["shared"] + m + t for t in steps], dtype=torch.float64, device="cuda")[:, None] * freq
        z = torch.polar(torch.ones_like(a), a)[:, None]
        for heads, w in ((slice(0, Hq), s["qw"]), (slice(Hq, Hq + Hkv), s["kw"])):
            t = x[:, heads]
            if w is not None:
                t = t / (t.square().sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
            t = torch.complex(t[..., :D // 2], t[..., D // 2:]) * z
            x[:, heads] = torch.cat([t.real, t.imag], -1)
        q_out[first:first + n] = x[:, :Hq]
        for name, t in (("k", x[:, Hq:Hq + Hkv]), ("v", x[:, Hq + Hkv:])):
            codes, scales = pools[name], pools[name + "s"]
            at = 0
            while at < n:  # block by block
                token = m + at
                take = min(n - at, BLOCK - token % BLOCK)
                page, row = table[b][token // R], token % R
                lo = row // BLOCK * BLOCK
                e = _least(t[at:at + take].abs().amax((0, 2)))                     # [Hkv]
                held = row - lo if at == 0 else 0
                if held:
                    was = scales[page, :, lo // BLOCK].log2().round()
                    e = torch.maximum(e, was)
                    codes[page, :, lo:row] = _e4m3(codes[page, :, lo:row] * _two(was - e)[:, None, None])
                y = t[at:at + take].transpose(0, 1) / _two(e)[:, None, None]
                codes[page, :, row:row + take] = _e4m3(y.clamp(-448.0, 448.0))
                scales[page, :, lo // BLOCK] = _two(e)
                at += take
        first += n
    return {"q": q_out, **pools}


def _exact_attn8(c, s):
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["shared"]
    out = s["out"].double()

    def tokens(codes, scales, pages):  # [Hkv][tokens][D]
        parts = [codes[p].double() * scales[p].double().repeat_interleave(BLOCK, 1)[..., None] for p in pages]
        return torch.cat(parts, 1)

    pools = ((s["k"], s["ks"]), (s["v"], s["vs"]))
    sh = [tokens(*p, s["shared_pages"].tolist())[:, :S] for p in pools] if S else [None, None]
    words = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    first = 0
    for b, (n, m) in enumerate(zip(s["rows"], s["lens"])):
        ids = s["table"][b, :(n + m + c["page"] - 1) // c["page"]].tolist()
        K, V = (tokens(*p, ids)[:, :n + m] for p in pools)
        allowed = np.ones((n, S + m + n), bool)
        if words is None:
            allowed[:, S + m:] = np.tri(n, dtype=bool)
        else:
            w = words[first:first + n]
            allowed[:, S + m:] = [[bool(int(w[i, j // 64]) >> (j % 64) & 1) for j in range(n)] for i in range(n)]
        allowed = torch.from_numpy(allowed).cuda()
        q = s["q"][first:first + n].double()
        for g in range(Hkv):
            kg = K[g] if not S else torch.cat([sh[0][g], K[g]])
            vg = V[g] if not S else torch.cat([sh[1][g], V[g]])
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                x = (q[:, h] @ kg.t()) * s["scale"]
                out[first:first + n, h] = torch.softmax(x.masked_fill(~allowed, -math.inf), -1) @ vg
        first += n
    return out


def _exact_compact8(c, s):
    R = c["page"]
    pools = {n: s[n].double() for n in ("k", "v", "ks", "vs")}
    table = s["table"].tolist()
    for b, m in enumerate(s["lens"]):
        path = s["path"][b, :int(s["accept"][b]) + 1].tolist()
        place = [(table[b][(m + i) // R], (m + i) % R) for i in range(s["rows"][b])]
        for name in ("k", "v"):
            codes, scales = pools[name], pools[name + "s"]
            at = 0
            while at < len(path):  # destination blocks in turn: their sources lie in them or behind them
                page, row = place[at]
                take = min(len(path) - at, BLOCK - row % BLOCK)
                lo, held = row // BLOCK * BLOCK, row % BLOCK
                src = [place[i] for i in path[at:at + take]]
                x = torch.stack([codes[:, p, :, r] for p, r in src], 2)                     # [L][Hkv][take][D]
                e = torch.stack([scales[:, p, :, r // BLOCK] for p, r in src], 2).log2().round()    # [L][Hkv][take]
                top = e.amax(2)
                if held:
                    was = scales[:, page, :, lo // BLOCK].log2().round()
                    top = torch.maximum(top, was)
                    codes[:, page, :, lo:row] = _e4m3(codes[:, page, :, lo:row]
                                                      * _two(was - top)[..., None, None])
                codes[:, page, :, row:row + take] = _e4m3(x * _two(e - top[..., None])[..., None])
                scales[:, page, :, lo // BLOCK] = _two(top)
                at += take
    return pools
