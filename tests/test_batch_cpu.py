"""The batch's entry points on the CPU: declarations, refusals before any
device work, and the reference's own pins."""

import ctypes
import os
import re

import numpy as np
import pytest

from oracle import batch as ob
from paper_2608_00814_amd import ooo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KEPT = []
P = 0x10000  # an address that is never read: refusals come first


def struct(**kw):
    b = ooo.PagedBatchStruct()
    KEPT.append(b)  # callers hold its address alone
    d = dict(n_seqs=2, n_rows=4, row_start=P, seq_len=P, page_table=P, shared_pages=P, anc_mask=None,
             page_stride=8 * 64 * 128, table_ld=4, shared_len=100, page_rows=64, n_pages=16, n_q_heads=32,
             n_kv_heads=8, head_dim=128, mask_words=0, dt=ooo.BF16)
    d.update(kw)
    for k, v in d.items():
        setattr(b, k, v)
    return b


def test_declared_and_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ooo_batch.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ooo_[a-z_0-9]+)\s*\(", text))
    assert names == set(ooo.BATCH_SIGNATURES)
    for n in names:
        assert getattr(ooo.lib(), n) is not None


BAD = [
    (dict(n_seqs=0), ooo.ERR_INVALID), (dict(n_rows=0), ooo.ERR_INVALID), (dict(row_start=None), ooo.ERR_INVALID),
    (dict(seq_len=None), ooo.ERR_INVALID), (dict(page_table=None), ooo.ERR_INVALID),
    (dict(shared_pages=None), ooo.ERR_INVALID), (dict(shared_len=-1), ooo.ERR_INVALID),
    (dict(table_ld=0), ooo.ERR_INVALID), (dict(n_pages=0), ooo.ERR_INVALID), (dict(n_q_heads=30), ooo.ERR_INVALID),
    (dict(n_kv_heads=0), ooo.ERR_INVALID), (dict(dt=5), ooo.ERR_INVALID), (dict(mask_words=1), ooo.ERR_INVALID),
    (dict(anc_mask=P, mask_words=0), ooo.ERR_INVALID), (dict(anc_mask=P, mask_words=17), ooo.ERR_INVALID),
    (dict(page_stride=8 * 64 * 128 - 8), ooo.ERR_INVALID), (dict(page_stride=8 * 64 * 128 + 4), ooo.ERR_UNSUPPORTED),
    (dict(head_dim=96), ooo.ERR_UNSUPPORTED), (dict(page_rows=48), ooo.ERR_UNSUPPORTED),
    (dict(page_rows=8), ooo.ERR_UNSUPPORTED), (dict(n_seqs=70000), ooo.ERR_UNSUPPORTED),
    (dict(n_rows=1 << 27), ooo.ERR_UNSUPPORTED), (dict(table_ld=1 << 25), ooo.ERR_UNSUPPORTED),
]


def calls(b):
    a = ctypes.addressof(b)
    L = ooo.lib()
    yield L.ooo_paged_append(a, P, 48 * 128, None, None, 1e-6, None, 1e6, 2 * P, P, P, None)
    yield L.ooo_paged_plan(a, P, 1 << 40, None)
    yield L.ooo_paged_attn(a, P, 1 << 40, P, P, P, 0.1, P, P, 1 << 40, None)
    yield L.ooo_paged_compact(a, P, P, 1, 0, P, P, 8, None)


@pytest.mark.parametrize("kw,status", BAD, ids=[str(k) for k, _ in BAD])
def test_bad_batches(kw, status):
    b = struct(**kw)
    for rc in calls(b):
        assert rc == status, ooo.last_error()
        assert ooo.last_error()
    assert ooo.lib().ooo_paged_plan_bytes(ctypes.addressof(b)) == 0
    assert ooo.lib().ooo_paged_attn_workspace(ctypes.addressof(b)) == 0


@pytest.mark.parametrize("kw", [dict(n_seqs=65536),
                                dict(anc_mask=P, mask_words=16, n_rows=1 << 25, n_q_heads=8, n_kv_heads=8)])
def test_sizes_past_the_kernels_offsets(kw):
    for rc in calls(struct(**kw)):
        assert rc == ooo.ERR_UNSUPPORTED, ooo.last_error()


def test_sample_rows_and_alignment():
    L = ooo.lib()
    s = lambda n=4, w=P: L.ooo_sample(P, 1000, ooo.F32, n, 1000, None, None, None, None, P, P, None, None, w,  # noqa: E731
                                      1 << 40, None)
    assert s(n=65536) == s(w=P + 8) == ooo.ERR_UNSUPPORTED


def test_null_batch():
    L = ooo.lib()
    assert L.ooo_paged_plan(None, P, 64, None) == ooo.ERR_INVALID
    assert L.ooo_paged_plan_bytes(None) == 0 and L.ooo_paged_attn_workspace(None) == 0


def test_append_refusals():
    a, L = ctypes.addressof(struct()), ooo.lib()
    f = lambda qkv=P, ld=48 * 128, qn=None, eps=1e-6, theta=1e6, q=P, k=P: L.ooo_paged_append(  # noqa: E731
        a, qkv, ld, qn, None, eps, None, theta, q, k, P, None)
    assert f(qkv=None) == f(q=None) == f(k=None) == ooo.ERR_INVALID
    assert f(ld=48 * 128 - 8) == f(eps=-1.0) == f(theta=0.0) == ooo.ERR_INVALID
    assert f(ld=48 * 128 + 4) == f(qkv=P + 2) == f(qn=P + 8) == f(k=P + 8) == ooo.ERR_UNSUPPORTED


def test_attn_and_plan_refusals():
    b = struct()
    a, L = ctypes.addressof(b), ooo.lib()
    plan, ws = L.ooo_paged_plan_bytes(a), L.ooo_paged_attn_workspace(a)
    assert plan > 0 and ws > 0
    assert L.ooo_paged_plan(a, None, plan, None) == ooo.ERR_INVALID
    assert L.ooo_paged_plan(a, P, plan - 1, None) == ooo.ERR_CAPACITY
    assert L.ooo_paged_plan(a, P + 4, plan, None) == ooo.ERR_UNSUPPORTED
    f = lambda pl=P, pb=plan, q=P, o=P, w=P, wb=ws: L.ooo_paged_attn(  # noqa: E731
        a, pl, pb, q, P, P, 0.1, o, w, wb, None)
    assert f(pl=None) == f(q=None) == f(o=None) == f(w=None) == ooo.ERR_INVALID
    assert f(pb=plan - 1) == f(wb=ws - 1) == ooo.ERR_CAPACITY
    assert f(q=P + 2) == f(w=P + 4) == ooo.ERR_UNSUPPORTED


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_attn_refuses_scales_that_are_not_finite(scale):
    """3e38 log2(e) is past the largest float32."""
    for dt in (ooo.BF16, ooo.F32):
        a, L = ctypes.addressof(struct(dt=dt)), ooo.lib()
        assert L.ooo_paged_attn(a, P, 1 << 40, P, P, P, scale, P, P, 1 << 40, None) == ooo.ERR_INVALID
        assert "scale" in ooo.last_error()


def test_calls_are_for_the_current_device(monkeypatch):
    import torch

    class Stream:
        def __init__(self, device):
            self.device, self.cuda_stream = torch.device(device), 77

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 100 + d, raising=False)
    on = lambda d, s: ooo._stream_on(torch.device("cuda", d), s)  # noqa: E731
    assert on(1, None) == 101 and on(1, 5) == 5 and on(1, Stream("cuda:1")) == 77
    for s in (None, 5, Stream("cuda:0"), Stream("cuda:1")):
        with pytest.raises(ValueError, match="current device"):
            on(0, s)
    with pytest.raises(ValueError, match="the stream is on"):
        on(1, Stream("cuda:0"))


def test_size_queries_follow_sizes_alone():
    """More rows, sequences or shared tokens never need less."""
    L = ooo.lib()
    size = lambda **kw: (L.ooo_paged_plan_bytes(ctypes.addressof(struct(**kw))),  # noqa: E731
                         L.ooo_paged_attn_workspace(ctypes.addressof(struct(**kw))))
    for key, values in (("n_rows", (1, 2, 7, 64, 1000, 8192)), ("n_seqs", (1, 3, 64, 1024))):
        got = [size(**{key: v}) for v in values]
        assert got == sorted(got) and all(x > 0 for g in got for x in g)


def test_compact_and_sample_refusals():
    a, L = ctypes.addressof(struct()), ooo.lib()
    f = lambda k=P, n=1, st=0, path=P, cap=8: L.ooo_paged_compact(a, k, P, n, st, path, P, cap, None)  # noqa: E731
    assert f(k=None) == f(path=None) == f(n=0) == f(cap=0) == f(n=2, st=0) == ooo.ERR_INVALID
    assert f(k=P + 8) == f(n=2, st=4) == ooo.ERR_UNSUPPORTED
    ws = L.ooo_sample_workspace(4, 1000)
    assert ws > 0 and L.ooo_sample_workspace(0, 10) == L.ooo_sample_workspace(1, 0) == 0
    assert L.ooo_sample_workspace(1, (1 << 20) + 1) == 0
    s = lambda x=P, ld=1000, dt=ooo.F32, n=4, V=1000, u=P, ids=P, w=P, wb=ws: L.ooo_sample(  # noqa: E731
        x, ld, dt, n, V, None, None, None, None, u, ids, None, None, w, wb, None)
    assert s(x=None) == s(u=None) == s(ids=None) == s(w=None) == ooo.ERR_INVALID
    assert s(n=0) == s(V=0) == s(ld=999) == s(dt=7) == ooo.ERR_INVALID
    assert s(wb=ws - 1) == ooo.ERR_CAPACITY
    assert s(V=(1 << 20) + 1, ld=1 << 21) == ooo.ERR_UNSUPPORTED


# --------------------------------------------------------------- the oracle


def test_sample_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))  # order: 1, 3, 4, 0, 2
    at = lambda **kw: ob.sample(x, **{**dict(T=1.0, k=0, top_p=1.0, min_p=0.0, u=0.0), **kw})  # noqa: E731
    assert at()[0] == 1 and at(u=0.39)[0] == 1 and at(u=0.41)[0] == 3 and at(u=0.66)[0] == 4
    assert at(u=0.81)[0] == 0 and at(u=0.95)[0] == 2 and at()[2] == 5
    assert at(k=2, u=0.62)[0] == 3 and at(k=2, u=0.61)[0] == 1 and at(k=2)[2] == 2
    assert at(top_p=0.6)[2] == 2 and at(top_p=0.7)[2] == 3 and at(top_p=0.0)[2] == 1
    assert at(k=2, top_p=0.6)[2] == 1  # 0.4 of 0.65 reaches 0.6
    assert at(min_p=0.3)[2] == 3 and at(min_p=0.7)[2] == 1 and at(min_p=5.0)[2] == 1
    assert at(T=0.0, u=0.99) == (1, 1.0, 1)
    assert ob.sample(np.array([-np.inf, np.nan]), 1.0, 0, 1.0, 0.0, 0.5) == (-1, 0.0, 0)
    assert ob.sample(np.array([1.0, np.inf, np.inf]), 1.0, 0, 1.0, 0.0, 0.6)[0] == 2


def test_visible_and_place():
    assert ob.visible(2, 5, None) == [0, 1, 2]
    assert ob.visible(2, 5, [0b10110]) == [1, 2, 4] and ob.visible(0, 2, [0b10110]) == [1]
    assert ob.visible(0, 70, [0, 1 << 3]) == [67]
    assert ob.place([9, 4], 17, 16) == (4, 1)


def test_attention_of_one_key_is_its_value():
    o, A, _ = ob.attention_row(np.ones(4), np.ones((1, 4)), np.array([[1.0, -2.0, 3.0, 4.0]]), 0.5)
    assert np.allclose(o, [1, -2, 3, 4]) and np.allclose(A, [1, 2, 3, 4])
    assert not ob.attention_row(np.ones(4), np.ones((0, 4)), np.ones((0, 4)), 0.5)[0].any()
