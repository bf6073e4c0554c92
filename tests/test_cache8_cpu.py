"""The 8-bit cache's entry points on the CPU: declarations, refusals before any
device work, and the reference's own pins."""

import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import cache8 as oc
from paper_2608_00814_amd import ooo
from test_batch_cpu import BAD, P, struct

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KEPT = []


def batch8(**kw):
    return ctypes.addressof(struct(**{**dict(page_stride=8 * 64 * 128), **kw}))


def cache8(**kw):
    c = ooo.Cache8Struct()
    KEPT.append(c)
    d = dict(k_pages=P, v_pages=P, k_scales=P + 1, v_scales=P + 3, layer_stride=1 << 20, scale_stride=16,
             scale_layer_stride=999, n_layers=2)
    d.update(kw)
    for k, v in d.items():
        setattr(c, k, v)
    return ctypes.addressof(c)


def calls(a, c):
    L = ooo.lib()
    yield L.ooo_paged_append8(a, c, 0, P, 48 * 128, None, None, 1e-6, None, 1e6, 2 * P, None)
    yield L.ooo_paged_attn8(a, c, 0, P, 1 << 40, P, 0.1, P, P, 1 << 40, None)
    yield L.ooo_paged_compact8(a, c, P, P, 8, None)
    yield L.ooo_paged_fork8(a, c, P, P, 2 * P, 2 * P, None)


def test_declared_and_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ooo_cache8.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ooo_[a-z_0-9]+)\s*\(", text))
    assert names == set(ooo.CACHE8_SIGNATURES)
    for n in names:
        assert getattr(ooo.lib(), n) is not None


BAD8 = BAD + [(dict(page_rows=16, page_stride=8 * 16 * 128), ooo.ERR_UNSUPPORTED),
              (dict(page_stride=8 * 64 * 128 + 8), ooo.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD8, ids=[str(k) for k, _ in BAD8])
def test_bad_batches(kw, status):
    a, L = batch8(**kw), ooo.lib()
    for rc in (*calls(a, cache8()), L.ooo_paged_plan8(a, P, 1 << 40, None)):
        assert rc == status, ooo.last_error()
        assert ooo.last_error()
    assert L.ooo_paged_plan8_bytes(a) == 0 and L.ooo_paged_attn8_workspace(a) == 0
    if (kw, status) in BAD:
        assert L.ooo_paged_fork(a, P, P, 1, 0, P, P, 2 * P, 2 * P, None) == status


BADC = [(dict(k_pages=None), ooo.ERR_INVALID), (dict(v_pages=None), ooo.ERR_INVALID),
        (dict(k_scales=None), ooo.ERR_INVALID), (dict(v_scales=None), ooo.ERR_INVALID),
        (dict(n_layers=0), ooo.ERR_INVALID), (dict(scale_stride=15), ooo.ERR_INVALID),
        (dict(layer_stride=0), ooo.ERR_INVALID), (dict(scale_layer_stride=0), ooo.ERR_INVALID),
        (dict(layer_stride=(1 << 20) + 8), ooo.ERR_UNSUPPORTED), (dict(k_pages=P + 8), ooo.ERR_UNSUPPORTED),
        (dict(n_layers=65536), ooo.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BADC, ids=[str(k) for k, _ in BADC])
def test_bad_caches(kw, status):
    for rc in calls(batch8(), cache8(**kw)):
        assert rc == status, ooo.last_error()


def test_null_and_layers():
    a, c, L = batch8(), cache8(), ooo.lib()
    for rc in (*calls(a, None), *calls(None, c)):
        assert rc == ooo.ERR_INVALID
    assert L.ooo_paged_plan8(None, P, 64, None) == ooo.ERR_INVALID
    for layer in (-1, 2):
        assert L.ooo_paged_append8(a, c, layer, P, 48 * 128, None, None, 1e-6, None, 1e6, 2 * P,
                                   None) == ooo.ERR_INVALID
        assert L.ooo_paged_attn8(a, c, layer, P, 1 << 40, P, 0.1, P, P, 1 << 40, None) == ooo.ERR_INVALID


def test_append_refusals():
    a, c, L = batch8(), cache8(), ooo.lib()
    f = lambda qkv=P, ld=48 * 128, qn=None, eps=1e-6, theta=1e6, q=P: L.ooo_paged_append8(  # noqa: E731
        a, c, 0, qkv, ld, qn, None, eps, None, theta, q, None)
    assert f(qkv=None) == f(q=None) == ooo.ERR_INVALID
    assert f(ld=48 * 128 - 8) == f(eps=-1.0) == f(theta=0.0) == ooo.ERR_INVALID
    assert f(ld=48 * 128 + 4) == f(qkv=P + 2) == f(qn=P + 8) == f(q=P + 8) == ooo.ERR_UNSUPPORTED
    # more rows than one launch has threads for (rows/8 + rows/4 workgroups of 256)
    one = dict(n_q_heads=1, n_kv_heads=1, head_dim=64, page_stride=64 * 64)
    many = batch8(**one, n_rows=(1 << 32) // 96 + 32)
    assert L.ooo_paged_append8(many, c, 0, P, 3 * 64, None, None, 1e-6, None, 1e6, 2 * P, None) == ooo.ERR_UNSUPPORTED
    assert b"threads" in L.ooo_last_error()


def test_attn_and_plan_refusals():
    a, c, L = batch8(), cache8(), ooo.lib()
    plan, ws = L.ooo_paged_plan8_bytes(a), L.ooo_paged_attn8_workspace(a)
    assert plan > 0 and ws > 0
    assert L.ooo_paged_plan8(a, None, plan, None) == ooo.ERR_INVALID
    assert L.ooo_paged_plan8(a, P, plan - 1, None) == ooo.ERR_CAPACITY
    assert L.ooo_paged_plan8(a, P + 4, plan, None) == ooo.ERR_UNSUPPORTED
    f = lambda pl=P, pb=plan, q=P, o=P, w=P, wb=ws, s=0.1: L.ooo_paged_attn8(  # noqa: E731
        a, c, 0, pl, pb, q, s, o, w, wb, None)
    assert f(pl=None) == f(q=None) == f(o=None) == f(w=None) == ooo.ERR_INVALID
    assert f(s=float("nan")) == f(s=float("inf")) == f(s=3e38) == ooo.ERR_INVALID
    assert f(pb=plan - 1) == f(wb=ws - 1) == ooo.ERR_CAPACITY
    assert f(q=P + 2) == f(w=P + 4) == ooo.ERR_UNSUPPORTED


def test_compact_and_fork_refusals():
    a, c, L = batch8(), cache8(), ooo.lib()
    assert L.ooo_paged_compact8(a, c, None, P, 8, None) == ooo.ERR_INVALID
    assert L.ooo_paged_compact8(a, c, P, None, 8, None) == ooo.ERR_INVALID
    assert L.ooo_paged_compact8(a, c, P, P, 0, None) == ooo.ERR_INVALID
    f8 = lambda p=P, f=P, n=2 * P, t=2 * P: L.ooo_paged_fork8(a, c, p, f, n, t, None)  # noqa: E731
    f = lambda p=P, f=P, n=2 * P, t=2 * P, k=P, nl=1, st=0: L.ooo_paged_fork(  # noqa: E731
        a, k, P, nl, st, p, f, n, t, None)
    for call in (f8, f):
        assert call(p=None) == call(f=None) == call(n=None) == call(t=None) == ooo.ERR_INVALID
        assert call(n=P) == call(t=P) == ooo.ERR_INVALID  # one of the two in place (the batch's are at P)
        assert "both" in ooo.last_error()
    assert f(k=None) == f(nl=0) == f(nl=2, st=0) == ooo.ERR_INVALID
    assert f(k=P + 8) == f(nl=2, st=4) == f(nl=65536, st=8) == ooo.ERR_UNSUPPORTED


# --------------------------------------------------------------- the oracle


def test_numbers_are_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.NUMBERS, want, equal_nan=True)
    assert oc.NUMBERS[126] == 448.0 and oc.NUMBERS[1] == 2.0 ** -9


def test_rounding_is_the_types():
    r = np.random.default_rng(1)
    x = np.concatenate([oc.NUMBERS[:127], (oc.NUMBERS[:126] + oc.NUMBERS[1:127]) / 2,
                        r.standard_normal(5000) * np.exp2(r.uniform(-12, 8, 5000))]).astype(np.float32)
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(oc.round8(x), want)
    assert oc.round8(np.array([1e9, -500.0, np.inf, np.nan])).tolist() == [126, 254, 127, 127]


def test_exponents_by_hand():
    assert oc.exponent(448.0) == 0 and oc.exponent(448.0000001) == 1 and oc.exponent(224.0) == -1
    assert oc.exponent(0.0) == oc.exponent(1e-40) == -100 and oc.exponent(3e38) == 119
    assert oc.exponent(1.0) == -8 and oc.exponent(1.75) == -8 and oc.exponent(1.7500001) == -7


def test_append_by_hand():
    """A block of one head: two committed rows, a small new one, then a large one."""
    codes, scales = np.zeros((1, 1, 32, 2), np.uint8), np.full((1, 1, 1), 127, np.uint8)
    codes[0, 0, :2] = oc.round8(np.array([[1.0, 3.0], [0.25, 2.0 ** -9 * 3]]))
    oc.append(codes, scales, np.array([[[5.0, 100.0]]]), [0], 2, 32)
    assert scales[0, 0, 0] == 127  # no less than it was
    assert oc.values(codes, scales)[0, 0, :3].tolist() == [[1, 3], [0.25, 2.0 ** -9 * 3], [5, 96]]  # 12.5 steps of 8: to 12
    oc.append(codes, scales, np.array([[[800.0, 1.0]]]), [0], 3, 32)
    assert scales[0, 0, 0] == 128
    # 3 2^-9 under twice the scale lies between 1 and 2 of the least number: even
    assert oc.values(codes, scales)[0, 0, :4].tolist() == [[1, 3], [0.25, 2.0 ** -9 * 4], [5, 96], [768, 1]]


def test_compact_by_hand():
    """Rows of two blocks of other scales meet; rows that are not moved keep their bytes."""
    codes, scales = np.zeros((3, 1, 32, 1), np.uint8), np.array([[[127]], [[130]], [[126]]], np.uint8)
    codes[:, 0, :, 0] = oc.round8(np.arange(1, 33))[None]
    c, s = oc.compact(codes, scales, [0, 40], [30], [[0, 1, 2]], np.array([[0, 1, 4, 39, -1]]), [3], 32)
    assert s.ravel().tolist() == [127, 130, 126]
    v, old = oc.values(c, s), oc.values(codes, scales)
    assert v[1, 0, 0, 0] == old[1, 0, 2, 0] and v[1, 0, 1, 0] == oc.NUMBERS[oc.round8(old[2, 0, 5, 0] / 8)] * 8
    assert np.array_equal(c[0], codes[0]) and np.array_equal(c[1, :, 2:], codes[1, :, 2:])
    # one row from a block of a larger scale into an open block: its committed rows are put under it
    c, s = oc.compact(codes, scales, [0, 40], [30], [[0, 1, 2]], np.array([[0, 4]]), [1], 32)
    assert s.ravel().tolist() == [130, 130, 126]
    assert np.array_equal(oc.values(c, s)[0, 0, :31], oc.values(codes, scales)[0, 0, :31])  # nothing was subnormal


def test_fork_by_hand():
    table = np.array([[4, 5, 6], [7, 8, 9], [1, 2, 3]])
    n, t, c = oc.fork([40, 7, 32], table, [-1, 0, 0], [-1, 10, 11], 12, 32, True)
    assert n.tolist() == [40, 40, 40] and t.tolist() == [[4, 5, 6], [4, 10, 9], [4, 11, 3]]
    assert c == [(1, 5, 10, 8), (2, 5, 11, 8)]
    n, t, c = oc.fork([40, 7, 32], table, [2, 0, -1], [0, 10, 11], 12, 32, True)
    assert n.tolist() == [32, 7, 32] and t.tolist() == [[1, 0, 6], [7, 8, 9], [1, 2, 3]] and c == []
    n, t, c = oc.fork([40, 7, 32], table, [1, 0, 9], [0, 10, 11], 12, 32, False)  # two change places
    assert n.tolist() == [7, 40, 32] and t.tolist() == [[0, 5, 6], [4, 10, 9], [1, 2, 3]]
    assert c == [(0, 7, 0, 7), (1, 5, 10, 8)]
