"""The operators of a batched step that are measured, with their plain forms.

A batch of requests shares one long tool prompt, keeps its other keys and
values in cache pages and samples its tokens: appending rows to the pages with
the head norms and the rotation (``append``), attention over the shared prompt
and each sequence's own pages (``attn``), moving the accepted rows of a batch
of tries together (``compact``) and drawing tokens from logits (``sample``).

Sizes are the repository's workload shapes (``workload.py``: 32 query and 8
KV heads of 128, 16 and 8, 40 and 8, one KV head of 64 in float32; prompts of
128 to 32768 rows; tries of 25 to 256 nodes; vocabularies of 1024 to 152064)
and generic ones.  A case's ``mix`` fixes its ragged lengths and tries; the
values come from the seed.
"""

import math
import random

import numpy as np
import torch

own = False

EPS = 1.0e-6
THETA = 1.0e6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # A float32 trie step of one small request: latency of the smallest append.
        {"name": "append_f32_trie", "kind": "append", "dt": "f32", "Hq": 4, "Hkv": 1, "D": 64, "seqs": 1, "rows": 25,
         "ragged": False, "trie": True, "shared": 128, "own": 64, "page": 16, "norm": True, "pad": 0, "mix": 1},
        # Prompts of 16 requests coming in at once, ragged, behind a common prefix: the bandwidth of an append.
        {"name": "append_prompts", "kind": "append", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 16,
         "rows": 1024, "ragged": True, "trie": False, "shared": 4096, "own": 512, "page": 64, "norm": True, "pad": 37,
         "mix": 2},
        # Float32 tries of three requests over a short prompt: the float32 option, small.
        {"name": "attn_f32_tries", "kind": "attn", "dt": "f32", "Hq": 4, "Hkv": 1, "D": 64, "seqs": 3, "rows": 25,
         "ragged": True, "trie": True, "shared": 128, "own": 100, "page": 16, "pad": 0, "mix": 3},
        # Plain decoding of 64 requests over a 4k tool prompt: the ordinary serving step.
        {"name": "attn_decode_64", "kind": "attn", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 64, "rows": 1,
         "ragged": False, "trie": False, "shared": 4096, "own": 1024, "page": 64, "pad": 0, "mix": 4},
        # Eight requests verifying tries of up to 64 nodes over the same prompt: the batched verify step.
        {"name": "attn_tries_8", "kind": "attn", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 8, "rows": 64,
         "ragged": True, "trie": True, "shared": 4096, "own": 512, "page": 32, "pad": 5, "mix": 5},
        # Chunks of four requests' own prompts, up to 512 rows each, behind a 1k prompt (Qwen3-0.6B heads).
        {"name": "attn_prompts_4", "kind": "attn", "dt": "bf16", "Hq": 16, "Hkv": 8, "D": 128, "seqs": 4, "rows": 512,
         "ragged": True, "trie": False, "shared": 1024, "own": 300, "page": 128, "pad": 0, "mix": 6},
        # 256 requests late in their calls over a 32k prompt, small pages: the largest step.
        {"name": "attn_decode_256", "kind": "attn", "dt": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "seqs": 256, "rows": 1,
         "ragged": False, "trie": False, "shared": 32768, "own": 2048, "page": 16, "pad": 0, "mix": 7},
        # One request's accepted float32 rows, one layer: the smallest commit.
        {"name": "compact_f32_one", "kind": "compact", "dt": "f32", "Hkv": 1, "D": 64, "layers": 1, "seqs": 1,
         "rows": 25, "own": 100, "page": 16, "mix": 8},
        # The commit of eight requests over all 36 layers.
        {"name": "compact_36x8", "kind": "compact", "dt": "bf16", "Hkv": 8, "D": 128, "layers": 36, "seqs": 8,
         "rows": 64, "own": 512, "page": 32, "mix": 9},
        # Logits of one small trie over a 1024-token vocabulary: the smallest draw.
        {"name": "sample_25x1k", "kind": "sample", "dt": "f32", "rows": 25, "vocab": 1024, "params": "mixed", "mix": 10},
        # The next token of one request.
        {"name": "sample_1", "kind": "sample", "dt": "f32", "rows": 1, "vocab": 151936, "params": "filtered", "mix": 11},
        # The next tokens of 256 requests with settings of their own.
        {"name": "sample_256", "kind": "sample", "dt": "f32", "rows": 256, "vocab": 152064, "params": "mixed",
         "mix": 12},
    ]


# ---------------------------------------------------------------- drawing


def _log(rng, lo, hi):
    """An integer between lo and hi, its logarithm spread evenly."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attn", "attn", "attn", "attn", "compact", "sample", "sample", "sample"])
    mix = rng.randrange(1 << 30)
    if kind == "sample":
        vocab = _log(rng, 500, 152064)
        rows = _log(rng, 1, 256)
        return {"kind": kind, "dt": rng.choice(["f32", "f32", "f32", "bf16"]), "rows": rows, "vocab": vocab,
                "params": rng.choice(["mixed", "mixed", "filtered", "plain"]), "mix": mix}
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "compact":
        return {"kind": kind, "dt": dt, "Hkv": rng.choice([1, 2, 4, 8]), "D": D, "layers": _log(rng, 1, 36),
                "seqs": _log(rng, 1, 8), "rows": _log(rng, 2, 64), "own": _log(rng, 1, 512), "page": page, "mix": mix}
    Hq, Hkv = rng.choice([(4, 1), (8, 8), (14, 2), (16, 8), (32, 8), (32, 8), (40, 8)])
    trie = rng.random() < 0.4
    common = {"kind": kind, "dt": dt, "Hq": Hq, "Hkv": Hkv, "D": D, "ragged": rng.random() < 0.7, "trie": trie}
    if kind == "append":
        rows = _log(rng, 1, 256 if trie else 1024)
        return {**common, "seqs": _log(rng, 1, max(1, min(256, 16384 // rows))), "rows": rows,
                "shared": _log(rng, 1, 32768), "own": _log(rng, 1, 2048), "page": page, "norm": rng.random() < 0.7,
                "pad": rng.choice([0, 0, 3, 50]), "mix": mix}
    rows = rng.choice([1, 1, _log(rng, 2, 256), _log(rng, 2, 256 if trie else 512)])
    seqs = _log(rng, 1, max(1, min(256, 2048 // rows)))
    shared = rng.choice([0, _log(rng, 16, 32768), _log(rng, 16, 32768)])
    own_len = _log(rng, 1, 2048)
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
        rows.append(r.randint(max(1, case["rows"] // 4), case["rows"]) if case.get("ragged") else case["rows"])
        lens.append(r.randint(case["own"] // 8, case["own"]))
    return rows, lens


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


def _batch(case, seed):
    """Page tables and lengths of a batch; the pool's pages are handed out in random order, two of them unused."""
    rows, lens = _lengths(case)
    R = case["page"]
    need = [(n + m + R - 1) // R for n, m in zip(rows, lens)]
    ns = (case.get("shared", 0) + R - 1) // R
    n_pages = sum(need) + ns + 2
    ids = np.random.default_rng(int(seed) % (1 << 32)).permutation(n_pages).astype(np.int32)
    table = np.zeros((len(rows), max(need)), np.int32)
    at = ns
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    total = sum(rows)
    return {"rows": rows, "lens": lens, "total": total, "n_rows": total + case.get("pad", 0), "n_pages": n_pages,
            "row_start": _dev(np.cumsum([0] + rows).astype(np.int32)), "seq_len": _dev(np.array(lens, np.int32)),
            "table": _dev(table), "shared_pages": _dev(ids[:ns]) if ns else None}


def prepare(case, seed):
    kind, dt = case["kind"], TYPES[case["dt"]]
    st = {"case": case}
    if kind == "sample":
        return _prepare_sample(case, seed, st)
    b = _batch(case, seed)
    st.update(b)
    R, Hkv, D = case["page"], case["Hkv"], case["D"]
    layers = (case["layers"],) if kind == "compact" else ()
    shape = layers + (b["n_pages"], Hkv, R, D)
    st["k"], st["v"] = _randn(shape, seed, 1, dt), _randn(shape, seed, 2, dt)
    n = b["n_rows"]
    if kind == "compact":
        r = random.Random(case["mix"] + 2 + seed)
        cap = max(b["rows"]) + 1
        path, acc = np.full((case["seqs"], cap), -1, np.int32), np.zeros(case["seqs"], np.int32)
        for s, m in enumerate(b["rows"]):  # a root path of the sequence's trie
            L = r.randint(0, m - 1)
            path[s, :L + 1] = [0] + sorted(r.sample(range(1, m), L))
            acc[s] = L
        st["path"], st["accept"] = _dev(path), _dev(acc)
    else:
        Hq = case["Hq"]
        st["mask"] = st["depth"] = None
        if case["trie"]:
            depth, mask = _tries(case, b["rows"])
            pad = n - b["total"]
            st["depth"] = _dev(np.concatenate([depth, np.zeros(pad, np.int32)]))
            st["mask"] = _dev(np.concatenate([mask, np.zeros((pad, mask.shape[1]), np.int64)]))
        if kind == "append":
            st["qkv"] = _randn((n, (Hq + 2 * Hkv) * D), seed, 3, dt)
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


def _prepare_sample(case, seed, st):
    n, V = case["rows"], case["vocab"]
    r = random.Random(case["mix"])
    T, k, p, m = [], [], [], []
    for _ in range(n):  # each request's own settings; "plain": temperature alone
        how = case["params"]
        how = r.choice(["greedy", "plain", "filtered", "filtered", "filtered"]) if how == "mixed" else how
        f = how == "filtered"
        T.append(0.0 if how == "greedy" else r.uniform(0.5, 1.3))
        k.append(r.choice([0, 20, 50, 200]) if f else 0)
        p.append(r.choice([1.0, 0.8, 0.9, 0.95]) if f else 1.0)
        m.append(r.choice([0.0, 0.0, 0.02, 0.1]) if f else 0.0)
    st["temperature"] = torch.tensor(T, dtype=torch.float32, device="cuda")
    st["top_k"] = torch.tensor(k, dtype=torch.int32, device="cuda")
    st["top_p"] = torch.tensor(p, dtype=torch.float32, device="cuda")
    st["min_p"] = torch.tensor(m, dtype=torch.float32, device="cuda")
    st["u"] = torch.rand(n, generator=_gen(seed, 1), device="cuda")
    x = _randn((n, V), seed, 2, torch.float32, 2.5)  # logits as a trained model's: a wide bulk, a few far above it
    x[:, torch.randint(V, (24,), generator=_gen(seed, 3), device="cuda")] += 6.0
    x[:, ::97] = float("-inf")                      # tokens that a grammar rules out
    st["logits"] = x.to(TYPES[case["dt"]])
    if own:
        from paper_2608_00814_amd import ooo

        st["ids"] = torch.empty(n, dtype=torch.int32, device="cuda")
        st["prob"] = torch.empty(n, dtype=torch.float32, device="cuda")
        st["kept"] = torch.empty(n, dtype=torch.int32, device="cuda")
        st["ws"] = torch.empty(ooo.sample_workspace(n, V), dtype=torch.uint8, device="cuda")
    return st


def _prepare_own(st):
    """What a serving program keeps: the batch's descriptor, the step's plan (one for all its layers) and scratch."""
    from paper_2608_00814_amd import ooo

    case = st["case"]
    pages = st["k"][0] if case["kind"] == "compact" else st["k"]
    st["batch"] = ooo.PagedBatch(st["row_start"], st["seq_len"], st["table"], pages, case.get("Hq", case["Hkv"]),
                                 n_rows=st["n_rows"], shared_pages=st["shared_pages"],
                                 shared_len=case.get("shared", 0), anc_mask=st.get("mask"))
    if case["kind"] == "attn":
        st["plan"] = ooo.paged_plan(st["batch"])
        st["ws"] = torch.empty(ooo.paged_attn_workspace(st["batch"]), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------- runs


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own[kind](state)
    return _plain[kind](state)


def _own_append(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_append(s["batch"], s["qkv"], s["qw"], s["kw"], EPS, THETA, s["q_out"], s["k"], s["v"], depth=s["depth"])
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _own_attn(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_attn(s["batch"], s["plan"], s["q"], s["k"], s["v"], s["scale"], s["out"], s["ws"])
    return s["out"]


def _own_compact(s):
    from paper_2608_00814_amd import ooo

    ooo.paged_compact(s["batch"], s["k"], s["v"], s["path"], s["accept"])
    return {"k": s["k"], "v": s["v"]}


def _own_sample(s):
    from paper_2608_00814_amd import ooo

    ooo.sample(s["logits"], s["u"], s["ids"], s["ws"], temperature=s["temperature"], top_k=s["top_k"],
               top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], kept=s["kept"])
    return {"ids": s["ids"], "prob": s["prob"], "kept": s["kept"]}


_own = {"append": _own_append, "attn": _own_attn, "compact": _own_compact, "sample": _own_sample}


def _rows_of(s):
    """Sequence and index in it of every row (rows behind the last sequence: those of row 0), and which are real."""
    r = torch.arange(s["n_rows"], device="cuda")
    real = r < s["row_start"][-1]
    r = torch.where(real, r, 0)
    b = torch.searchsorted(s["row_start"][1:].contiguous(), r.int(), right=True)
    return b, r - s["row_start"][b], real, r


def _plain_append(s):
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

    dt = s["qkv"].dtype
    page = s["table"][b, slot // R]
    s["k"][page, :, slot % R] = turned(k).to(dt)
    s["v"][page, :, slot % R] = v.to(dt)
    s["q_out"].copy_(torch.where(real[:, None, None], turned(q).to(dt), s["q_out"]))
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_attn(s):
    c = s["case"]
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["shared"]
    G, B, most = Hq // Hkv, c["seqs"], max(s["rows"])
    start, lens = s["row_start"][:-1].long(), s["seq_len"].long()
    count = s["row_start"][1:].long() - start
    i = torch.arange(most, device="cuda")
    at = torch.where(i < count[:, None], start[:, None] + i, 0)                     # [B][most]
    q = s["q"][at].float().view(B, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * G, D)
    kv = []
    for pages in (s["k"], s["v"]):
        t = pages[s["table"].long()].float()                                        # [B][pages][Hkv][R][D]
        kv.append(t.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D))
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
        shared = [p[s["shared_pages"].long()].float().transpose(0, 1).reshape(Hkv, -1, D)[:, :S] for p in (s["k"], s["v"])]
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


def _plain_compact(s):
    R = s["case"]["page"]
    d = torch.arange(s["path"].shape[1], device="cuda")
    on = d <= s["accept"][:, None]
    base = s["seq_len"][:, None]
    src = base + torch.where(on, s["path"], 0)
    dst = base + torch.where(on, d, 0)  # entries behind the path move the root to itself
    b = torch.arange(on.shape[0], device="cuda")[:, None].expand_as(src)
    sp, dp = s["table"][b, src // R], s["table"][b, dst // R]
    for t in (s["k"], s["v"]):
        t[:, dp, :, dst % R] = t[:, sp, :, src % R]
    return {"k": s["k"], "v": s["v"]}


def _plain_sample(s):
    x = s["logits"].double()
    V = x.shape[1]
    greedy = s["temperature"] <= 0
    T = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    live = (x > float("-inf")).sum(1)
    w = torch.exp((x - x[:, :1]) / T)
    k = torch.where(greedy, 1, torch.where(s["top_k"] > 0, s["top_k"], V)).long()
    k = torch.minimum(k, live)
    cum = torch.cumsum(w, 1)
    want = s["top_p"].double() * torch.gather(cum, 1, k[:, None] - 1)[:, 0]
    n_p = (cum < want[:, None]).sum(1) + 1
    n = torch.where(s["top_p"] < 1, torch.minimum(n_p, k), k)
    n_m = (w >= s["min_p"].double()[:, None]).sum(1).clamp_min(1)
    n = torch.where(s["min_p"] > 0, torch.minimum(n, n_m), n)
    total = torch.gather(cum, 1, n[:, None] - 1)
    at = torch.minimum((cum <= s["u"].double()[:, None] * total).sum(1), n - 1)[:, None]
    return {"ids": torch.gather(order, 1, at)[:, 0].int(), "prob": (torch.gather(w, 1, at) / total)[:, 0].float(),
            "kept": n.int()}


_plain = {"append": _plain_append, "attn": _plain_attn, "compact": _plain_compact, "sample": _plain_sample}


# ------------------------------------------------------------------- work


def work(case):
    kind, e = case["kind"], 4 if case["dt"] == "f32" else 2
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * e + 32 * case["rows"], "flops": 2.0 * n}
    rows, lens = _lengths(case)
    total, D, Hkv = sum(rows), case["D"], case["Hkv"]
    if kind == "compact":
        return {"bytes": 4.0 * case["layers"] * total / 2 * Hkv * D * e, "flops": 0}
    Hq = case["Hq"]
    if kind == "append":
        n = total * (Hq + 2 * Hkv) * D
        return {"bytes": 2.0 * n * e, "flops": 8.0 * n}
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
    return {"bytes": float(e) * (2 * total * Hq * D + 2 * Hkv * D * (case["shared"] + own_keys)),
            "flops": 4.0 * Hq * D * (seen + total * case["shared"])}


# ------------------------------------------------------------------ exact


def exact(case, seed):
    """The definitions in 64 bits, one sequence (or row) after the other."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "compact":
        return None  # rows are moved, nothing is computed
    return {"append": _exact_append, "attn": _exact_attn, "sample": _exact_sample}[kind](case, s)


def _exact_append(c, s):
    Hq, Hkv, D, R = c["Hq"], c["Hkv"], c["D"], c["page"]
    q_out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
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
        pages = torch.tensor([table[b][(m + i) // R] for i in range(n)], device="cuda")
        slots = torch.tensor([(m + i) % R for i in range(n)], device="cuda")
        k[pages, :, slots] = x[:, Hq:Hq + Hkv]
        v[pages, :, slots] = x[:, Hq + Hkv:]
        first += n
    return {"q": q_out, "k": k, "v": v}


def _exact_attn(c, s):
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["shared"]
    out = s["out"].double()
    sh = [None, None]
    if S:
        sh = [torch.cat(list(p[s["shared_pages"].long()].double()), 1)[:, :S] for p in (s["k"], s["v"])]
    words = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    first = 0
    for b, (n, m) in enumerate(zip(s["rows"], s["lens"])):
        ids = s["table"][b, :(n + m + c["page"] - 1) // c["page"]].long()
        K, V = (torch.cat(list(p[ids].double()), 1)[:, :n + m] for p in (s["k"], s["v"]))
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


def _exact_sample(c, s):
    x = s["logits"].double().cpu().numpy()
    ids, prob, kept = [], [], []
    get = lambda n: s[n].double().cpu().numpy()  # noqa: E731
    T, k, p, m, u = get("temperature"), get("top_k"), get("top_p"), get("min_p"), get("u")
    for r in range(c["rows"]):
        live = np.flatnonzero(x[r] > -np.inf)
        order = live[np.lexsort((live, -x[r][live]))]
        if T[r] <= 0:
            order = order[:1]
        elif k[r] > 0:
            order = order[:int(k[r])]
        w = np.exp((x[r][order] - x[r][order[0]]) / (T[r] if T[r] > 0 else 1.0))
        n = len(w)
        if p[r] < 1:
            n = min(n, 1 + int(np.searchsorted(np.cumsum(w), p[r] * w.sum(), side="left")))
        if m[r] > 0:
            n = min(n, max(1, int((w >= m[r]).sum())))
        cum = np.cumsum(w[:n])
        at = min(n - 1, int(np.searchsorted(cum, u[r] * cum[-1], side="right")))
        ids.append(int(order[at]))
        prob.append(float(w[at] / cum[-1]))
        kept.append(n)
    return {"ids": torch.tensor(ids, dtype=torch.int32), "prob": torch.tensor(prob, dtype=torch.float64),
            "kept": torch.tensor(kept, dtype=torch.int32)}
