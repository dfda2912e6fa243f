"""CPU tests of the sampling operators: the oracle's cache against what has to hold of any, its tree attention against packed
attention, its verification against the distribution that it has to leave alone; what the library refuses, and the checks
that its kernels make on what device arrays say."""
import ctypes
import itertools
import os
import subprocess

import numpy as np
import pytest

from oracle import pp_oracle as orc
from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
OK, OFF1, OFF4 = ctypes.c_void_p(4096), ctypes.c_void_p(4097), ctypes.c_void_p(4100)


# ---------------------------------------------------------------- the oracle


def _content(b, s):
    return [np.stack([p[:, b.place(s, t)[0], :, b.place(s, t)[1]] for t in range(int(b.len[s]))]) for p in b.pools]


def test_oracle_cache_keeps_sequences_and_counts():
    rng = np.random.default_rng(0)
    pages, slots, cols, ps = 20, 12, 6, 4
    k, v = rng.standard_normal((2, 2, pages, 3, ps, 5))
    b = smp.Book(np.zeros((slots, cols)), np.zeros(slots), np.zeros(slots), np.zeros(pages), ps, k, v)
    assert b.reserve([0, 1, 0], [9, 5, 9]) == [0, 1]  # a slot named twice counts once
    assert list(b.held[:2]) == [3, 2] and list(b.table[0, :3]) == [0, 1, 2]
    b.len[:2] = [9, 5]
    want = [_content(b, s) for s in (0, 1)]
    assert b.fork([0, 0, 1, 1], [4, 5, 6, 0]) == [0, 1]  # slot 0 is not empty
    for s, w in ((4, want[0]), (5, want[0]), (6, want[1])):
        for x, y in zip(_content(b, s), w):
            np.testing.assert_array_equal(x, y)
    assert b.refs[0] == 3 and b.refs[2] == 1 and b.refs.sum() == b.held.sum()
    b.free([0, 0])
    assert b.refs.sum() == b.held.sum() and b.refs[0] == 2 and b.refs[2] == 0
    live = b.compact()
    assert live == (b.refs > 0).sum() and (b.refs[:live] > 0).all() and b.refs.sum() == b.held.sum()
    for s, w in ((4, want[0]), (5, want[0]), (6, want[1]), (1, want[1])):
        for x, y in zip(_content(b, s), w):
            np.testing.assert_array_equal(x, y)
    assert b.shared([4, 5, -1, 6, 1, 7], 3) == [2, 0] and b.shared([4], 1) == [0]
    before = b.refs.copy()
    assert b.reserve([7], [ps * cols + 1]) == [0, 1] and b.reserve([7, 8, 9, 10, 11], [ps * cols] * 5)[0] > 0
    np.testing.assert_array_equal(before, b.refs)
    old = int(b.len[4])
    assert b.reserve([4], [6]) == [0, 0]
    want = [p[:, b.place(4, old + 3)[0], :, b.place(4, old + 3)[1]].copy() for p in b.pools]
    assert b.accept([4, 4], [2, 1], [[0, 3], [0, 0]]) == [0, 1] and b.len[4] == old + 2
    for p, w in zip(b.pools, want):
        np.testing.assert_array_equal(p[:, b.place(4, old + 1)[0], :, b.place(4, old + 1)[1]], w)


def test_oracle_tree_attention_equals_packed_attention():
    """A chain behind a cached prompt is the end of a packed row; two branches of a tree are two responses."""
    rng = np.random.default_rng(1)
    P, N, hq, hkv, d, ps = 7, 3, 4, 2, 8, 4
    q, k, v = rng.standard_normal((P + 2 * N, hq, d)), *rng.standard_normal((2, P + 2 * N, hkv, d))
    O, L = orc.attn_fwd([0, P + 2 * N], [P], [2], [[P, P + N]], [[N, N]], q, k, v)
    k_pool, v_pool = np.full((2, 1, 5, hkv, ps, d), np.nan)
    b = smp.Book([[3, 1, 4, 0]], [P], [4], np.ones(5), ps, k_pool, v_pool)
    for t in range(P + 2 * N):
        b.append(0, 0, t - P, k[t], v[t])
    o, lse, *_ = smp.tree_attn(b, 0, [0], q[None, P:], [[-1, 0, 1, -1, 3, 4]])
    np.testing.assert_allclose(o[0], O[P:], atol=1e-12)
    np.testing.assert_allclose(lse, L[:, P:], atol=1e-12)
    assert smp.depths([-1, 0, 1, -1, 3, 4]) == [0, 1, 2, 0, 1, 2]


def _threshold(f):
    """The number below which f is true (f falls once from true to false on [0, 1])."""
    lo, hi = 0.0, 1.0
    if not f(lo):
        return 0.0
    for _ in range(48):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if f(mid) else (lo, mid)
    return lo if lo < 1 - 1e-12 else 1.0


@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("children", [1, 2, 3])
def test_oracle_verification_leaves_the_distribution(drafted, children):
    """Summed over all drafts and integrated over all numbers, the first new token is distributed as p."""
    rng = np.random.default_rng(children)
    V, N, T = 3, children + 1, 0.8
    target, draft = rng.standard_normal((2, 1, N, V)) * 1.5
    soft = lambda x: np.exp(x / T) / np.exp(x / T).sum()
    p, q = soft(target[0, 0]), soft(draft[0, 0])
    parents, got = [[-1] + [0] * children], np.zeros(V)
    drafts = itertools.product(range(V), repeat=children) if drafted else [(1, 0, 1)[:children]]
    for y in drafts:
        weight = np.prod(q[list(y)]) if drafted else 1.0
        tokens = np.array([[0, *y]])

        def first(u):
            c, t, path, _ = smp.verify(target, tokens, np.array([u]), draft if drafted else None, parents, None, [T], children)
            return (int(path[0, 1]) if c[0] > 1 else 0), int(t[0, 0])

        left = 1.0  # that no child has followed yet
        for j in range(1, N):
            chance = _threshold(lambda x: first([0.5] + [1.0] * (j - 1) + [x] + [1.0] * (N - 1 - j))[0] == j)
            got[y[j - 1]] += weight * left * chance
            left *= 1 - chance
        if left > 1e-9:
            ends = [_threshold(lambda x: first([x] + [1.0] * (N - 1))[1] <= t) for t in range(V - 1)] + [1.0]
            got += weight * left * np.diff([0.0] + ends)
    np.testing.assert_allclose(got, p, atol=1e-6)


# ---------------------------------------------------------------- refusals


def _desc(num_slots=4, max_pages=8, num_pages=32, page_size=16, table=OK, length=OK, held=OK, refs=OK):
    return ctypes.byref(pp._CacheDesc(num_slots, max_pages, num_pages, page_size, table, length, held, refs))


def test_cache_descriptor_refusals():
    L, n = pp.lib(), ctypes.c_size_t(0)
    size = lambda d, m=4: L.pp_cache_workspace_size(d, m, ctypes.byref(n))
    assert size(_desc()) == 0 and n.value > 0
    assert size(None) == 1 and L.pp_cache_workspace_size(_desc(), 4, None) == 1
    for bad in ({"num_slots": 0}, {"max_pages": 0}, {"num_pages": -1}, {"table": None}, {"length": None}, {"held": None},
                {"refs": None}, {"refs": OFF1}):
        assert size(_desc(**bad)) == 1, bad
    for bad in ({"page_size": 8}, {"page_size": 24}, {"page_size": 512}, {"num_slots": 1 << 20, "max_pages": 1 << 12},
                {"max_pages": 1 << 24, "page_size": 256}, {"num_pages": 1 << 30}):
        assert size(_desc(**bad)) == 3, bad
    assert size(_desc(), -1) == 1 and size(_desc(), 70000) == 3


def test_cache_call_refusals():
    L, big = pp.lib(), 1 << 30
    reserve = lambda d=None, n=2, s=OK, a=OK, st=OK, ws=OK, b=big: L.pp_cache_reserve(d or _desc(), n, s, a, st, ws, b, None)
    assert reserve(s=None) == 1 and reserve(a=None) == 1 and reserve(st=None) == 1 and reserve(a=OFF1) == 1
    assert reserve(ws=None) == 1 and reserve(ws=OFF4) == 1 and reserve(b=16) == 4
    fork = lambda dt=0, layers=2, hkv=2, d=64, k=OK, v=OK, st=OK, b=big: L.pp_cache_fork(
        _desc(), 2, OK, OK, dt, layers, hkv, d, k, v, st, OK, b, None)
    assert fork(dt=5) == 1 and fork(layers=-1) == 1 and fork(hkv=0) == 1 and fork(k=None) == 1 and fork(v=OFF4) == 1
    assert fork(st=None) == 1 and fork(d=96) == 3 and fork(layers=20000) == 3 and fork(hkv=5000) == 3 and fork(b=1) == 4
    assert L.pp_cache_free(_desc(), 2, None, None) == 1 and L.pp_cache_free(None, 2, OK, None) == 1
    assert L.pp_cache_free(_desc(), 0, None, None) == 0
    compact = lambda k=OK, live=OK, d=64, b=big: L.pp_cache_compact(_desc(), 0, 1, 2, d, k, OK, live, OK, b, None)
    assert compact(k=None) == 1 and compact(live=None) == 1 and compact(d=32) == 3 and compact(b=1) == 4
    accept = lambda n=2, N=8, c=OK, path=OK, k=OK, st=OK, b=big: L.pp_cache_accept(
        _desc(), n, OK, N, c, path, 0, 1, 2, 64, k, OK, st, OK, b, None)
    assert accept(c=None) == 1 and accept(k=None) == 1 and accept(st=None) == 1 and accept(N=0) == 1 and accept(path=OFF1) == 1
    assert accept(N=65) == 3 and accept(b=1) == 4
    assert L.pp_cache_shared(_desc(), 4, OK, 3, OK, None) == 1 and L.pp_cache_shared(_desc(), 4, OK, 2, None, None) == 1
    app = lambda N=2, rows=4, start=None, par=None, dt=0, hq=4, hkv=2, d=64, base=1e4, q=OK, k=OK, qr=OK, kp=OK, s=OK: \
        L.pp_cache_append(_desc(), 2, s, N, None, start, rows, par, dt, hq, hkv, d, base, q, k, OK, qr, kp, OK, None)
    assert app(N=0) == 1 and app(rows=3) == 1 and app(rows=-1, start=OK) == 1 and app(hq=3) == 1 and app(q=None) == 1
    assert app(qr=None) == 1 and app(k=None) == 1 and app(k=OFF4) == 1 and app(kp=None) == 1 and app(s=None) == 1
    assert app(base=-1.0) == 1 and app(base=float("inf")) == 1 and app(base=float("nan")) == 1 and app(dt=7) == 1
    assert app(d=80) == 3 and app(N=65, rows=200, par=OK) == 3
    assert app(N=2**31 - 1, rows=4, start=OK) == 3 and app(N=2**24 + 1, rows=4, start=OK) == 3


def test_tree_and_verify_refusals():
    L, big, n = pp.lib(), 1 << 40, ctypes.c_size_t(0)
    tree = lambda n=4, group=2, N=3, dt=0, hq=4, hkv=2, d=64, q=OK, o=OK, lse=OK, s=OK, sh=OK, ws=OK, b=big: L.pp_tree_attn_fwd(
        _desc(), n, s, group, sh, N, None, None, dt, hq, hkv, d, 0.0, q, OK, OK, o, lse, 0, ws, b, None)
    assert tree(q=None) == 1 and tree(o=OFF4) == 1 and tree(lse=OFF1) == 1 and tree(s=None) == 1 and tree(sh=OFF1) == 1
    assert tree(group=3) == 1 and tree(group=0) == 1 and tree(N=0) == 1 and tree(hq=3) == 1 and tree(hkv=0) == 1 and tree(dt=2) == 1
    assert tree(N=65) == 3 and tree(n=2050) == 3 and tree(d=256) == 3 and tree(hq=8192) == 3 and tree(b=64) == 4 and tree(ws=None) == 1
    assert tree(n=0) == 0
    assert tree(n=2048, N=64, hq=1024, hkv=1) == 3 and tree(n=2048, N=64, hq=1023, hkv=1, b=64) == 4  # 2^27 rows
    assert L.pp_tree_workspace_size(_desc(), 4, 2, 3, 0, 4, 2, 64, ctypes.byref(n)) == 0 and n.value > 0
    assert L.pp_tree_workspace_size(_desc(), 4, 2, 3, 0, 4, 2, 64, None) == 1
    ver = lambda n=4, N=3, V=100, dt=0, kids=1, tok=OK, t=OK, dr=None, temp=None, u=OK, oc=OK, b=big: L.pp_verify_draft(
        n, N, V, dt, kids, None, None, tok, t, dr, temp, u, oc, OK, OK, OK, OK, b, None)
    assert ver(t=None) == 1 and ver(t=OFF1) == 1 and ver(dr=OFF1) == 1 and ver(tok=None) == 1 and ver(u=None) == 1
    assert ver(oc=None) == 1 and ver(temp=OFF1) == 1 and ver(N=0) == 1 and ver(V=0) == 1 and ver(kids=0) == 1 and ver(dt=3) == 1
    assert ver(n=-1) == 1 and ver(N=65) == 3 and ver(n=2000, N=64) == 3 and ver(V=2**31 - 1) == 3 and ver(b=8) == 4 and ver(n=0) == 0
    assert L.pp_verify_workspace_size(4, 3, 100, 0, None) == 1
    assert pp.pp_verify_workspace_size(4, 3, 128256) > pp.pp_verify_workspace_size(4, 3, 100) > 0


def test_what_the_kernels_check(tmp_path):
    """CacheView's checks, which stand ahead of every address that a kernel forms from a device array, on the host."""
    src = tmp_path / "view.cpp"
    src.write_text('#include "pp_sample.h"\n'
                   'extern "C" int view_ok(int what, long long a, long long b) {\n'
                   '  pp::CacheView c{nullptr, nullptr, nullptr, nullptr, 4, 3, 7, 16, 4};\n'
                   '  return what == 0 ? c.has_slot((int)a) : what == 1 ? c.has_page((int)a) : c.sound(a, b);\n}\n')
    so = tmp_path / "view.so"
    r = subprocess.run([build.hipcc(), *build.COMMON, "-shared", str(src), "-o", str(so)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    L = ctypes.CDLL(str(so))
    ok = lambda what, a, b=0: bool(L.view_ok(what, ctypes.c_longlong(a), ctypes.c_longlong(b)))
    for what, n in ((0, 4), (1, 7)):
        for x in (-2**31, -1, 0, n - 1, n, 2**31 - 1):
            assert ok(what, x) == (0 <= x < n)
    for length in (-1, 0, 1, 16, 17, 48, 49, 2**31 - 1):
        for held in (-1, 0, 1, 3, 4, 2**31 - 1):
            assert ok(2, length, held) == (0 <= held <= 3 and 0 <= length <= 16 * held)
