"""GPU tests of cross attention against the 64-bit oracle, within derived bounds
(cross_check.py): types, head layouts, lengths from none to many, key ranges that leave
tokens empty, split axes, padding on both axes."""
import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

import cross_check

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _inputs(pack, enc, hq, hkv, d, dtype, seed):
    q = wl.randn((pack.total_tokens, hq, d), seed, dtype, "cpu")
    k = wl.randn((enc.total_states, hkv, d), seed + 1, dtype, "cpu")
    v = wl.randn((enc.total_states, hkv, d), seed + 2, dtype, "cpu")
    do = wl.randn((pack.total_tokens, hq, d), seed + 3, dtype, "cpu")
    # states past each row's length are never read
    real = np.zeros(enc.total_states, bool)
    for b in range(pack.num_rows):
        real[enc.enc_start[b]:enc.enc_start[b] + enc.enc_len[b]] = True
    pad = torch.from_numpy(~real)
    k[pad], v[pad] = float("nan"), float("nan")
    return q, k, v, do


def _run(pack, enc, x, begin=None, end=None, scale=0.0):
    q, k, v, do = (t.to(DEV) for t in x)
    keys = {"key_begin": None if begin is None else torch.tensor(begin, dtype=torch.int32, device=DEV),
            "key_end": None if end is None else torch.tensor(end, dtype=torch.int32, device=DEV)}
    f, b = pp.pp_cross_workspace_size(pack, enc, q.shape[1], k.shape[1], q.shape[2], pp._dtype_code(q))
    junk = lambda n: torch.full((max(n, 1),), 0xff, dtype=torch.uint8, device=DEV)  # NaN in every type
    nan = lambda t: torch.full_like(t, float("nan"))
    lse = torch.full((q.shape[1], q.shape[0]), float("nan"), device=DEV)
    o, lse = pp.pp_cross_attn_fwd(pack, enc, q, k, v, scale=scale, out=nan(q), lse=lse, ws=junk(f), **keys)
    grads = pp.pp_cross_attn_bwd(pack, enc, q, k, v, o, lse, do, scale=scale, dq=nan(q), dk=nan(k), dv=nan(v), ws=junk(b),
                                 **keys)
    torch.cuda.synchronize()
    return (o, lse, *grads)


def _check(pack, enc, x, begin=None, end=None, scale=None):
    got = _run(pack, enc, x, begin, end, scale or 0.0)
    u = U[x[0].dtype]
    q, k, v, do = (np.nan_to_num(t.double().numpy()) for t in x)
    args = pack.oracle_args()
    want = orc.cross_attn(*args, enc.enc_start, enc.enc_len, q, k, v, do, begin, end, scale)
    vis = orc.cross_visible(*args, enc.enc_len, begin, end)
    bar = cross_check.bounds(args, enc.enc_start, enc.enc_len, q, k, v, do, vis, u, scale)
    for name, g, w, b in zip(("o", "lse", "dq", "dk", "dv"), got, want, bar):
        g = g.double().cpu().numpy()
        assert np.isfinite(g).all(), name
        assert (g[b == 0] == 0).all(), (name, "what nothing sees or reads is 0")
        off = np.abs(g - w) - cross_check.allow(b, w, 2.0 ** -24 if name == "lse" else u)
        assert off.size == 0 or off.max() <= 0, (name, float(off.max()), float(np.abs(g - w).max()))


HEADS = [(4, 4, 64), (14, 2, 64), (8, 1, 128), (6, 2, 128), (32, 8, 128), (5, 5, 128), (71, 1, 64)]
DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_single_tokens(hq, hkv, d, dtype):
    pack = wl.make_pack([1, 1, 1, 0, 1, 2], [[]] * 6)
    enc = wl.make_enc([1, 33, 0, 5, 640, 129], pad=[0, 3, 7, 0, 1, 0])
    _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 10))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
def test_lengths_of_states(n, dtype):
    pack = wl.make_pack([5, 40], [[3, 1], [30, 0, 2]], pad=[2, 0])
    enc = wl.make_enc([n, n + 1])
    for hq, hkv, d in [(4, 2, 64), (4, 2, 128)]:
        _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 20 + n))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_ragged_rows(hq, hkv, d, dtype):
    pack = wl.make_pack([17, 0, 70, 1, 0, 9], [[3, 20], [4, 5], [1, 1, 1], [], [], [0, 65]], pad=[5, 0, 3, 130, 0, 1])
    enc = wl.make_enc([130, 64, 0, 1, 12, 300], pad=[0, 200, 5, 0, 0, 1])
    _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 40))


def _images(rng, pack, enc, most=4):
    """Key ranges as of several images in a text, with tokens that see nothing and wild values."""
    begin, end = np.zeros(pack.total_tokens, np.int64), np.zeros(pack.total_tokens, np.int64)
    for b in range(pack.num_rows):
        t0, t1, n = int(pack.row_start[b]), int(pack.row_start[b + 1]), int(enc.enc_len[b])
        edge = np.sort(rng.integers(0, n + 1, size=most + 1))
        img = np.sort(rng.integers(0, most + 1, size=t1 - t0)) - 1  # -1: ahead of the first
        lo, hi = edge[np.maximum(img, 0)], edge[np.maximum(img, 0) + 1]
        begin[t0:t1], end[t0:t1] = np.where(img < 0, n, lo), np.where(img < 0, 0, hi)
    wild = rng.integers(0, max(1, pack.total_tokens), size=3)
    begin[wild], end[wild] = -2 ** 31, 2 ** 31 - 1  # everything
    return begin, end


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 64), (6, 2, 128)])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_key_ranges(seed, hq, hkv, d, dtype):
    rng = np.random.default_rng(seed)
    pack = wl.make_pack([90, 33, 1, 0, 150], [[40, 3], [64], [1, 1], [7], []], pad=[1, 0, 60, 0, 3])
    enc = wl.make_enc([400, 70, 33, 129, 0], pad=[3, 0, 0, 64, 2])
    begin, end = _images(rng, pack, enc)
    _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 60 + seed), begin, end)


def test_arbitrary_ranges():
    """Ranges without any order: every row of a block its own."""
    rng = np.random.default_rng(5)
    pack, enc = wl.make_pack([200], [[31, 40]], pad=[2]), wl.make_enc([500])
    begin, end = rng.integers(-50, 550, size=(2, pack.total_tokens))
    for dtype in DTYPES:
        _check(pack, enc, _inputs(pack, enc, 4, 2, 64, dtype, 80), begin, end)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ranges", [False, True])
def test_split_keys(ranges, dtype):
    """Few rows over many keys: the keys are split over workgroups; the rows of one part may see nothing of it."""
    pack, enc = wl.make_pack([3, 1], [[], [1]], pad=[1, 0]), wl.make_enc([5000, 3300], pad=[7, 0])
    begin = end = None
    if ranges:
        begin, end = np.array([100, 0, 4800, 7, 0, 5]), np.array([1900, 0, 5000, 9, 3300, 64])
    for hq, hkv, d in [(8, 2, 128), (8, 8, 64)]:
        _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 90), begin, end)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ranges", [False, True])
def test_split_rows(ranges, dtype):
    """Many rows over few keys: dK and dV come from parts of the rows."""
    pack, enc = wl.make_pack([700], [[300, 77]], pad=[3]), wl.make_enc([77], pad=[100])
    begin = end = None
    if ranges:
        rng = np.random.default_rng(9)
        begin, end = _images(rng, pack, enc, 3)
    for hq, hkv, d in [(4, 2, 128), (3, 1, 64)]:
        _check(pack, enc, _inputs(pack, enc, hq, hkv, d, dtype, 100), begin, end)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows_stage_their_records(dtype):
    """More tiles than the launch's arguments hold."""
    rng = np.random.default_rng(3)
    n = rng.integers(0, 60, size=90).tolist()
    pack, enc = wl.make_pack(n, [[1]] * 90), wl.make_enc(rng.integers(0, 90, size=90).tolist())
    _check(pack, enc, _inputs(pack, enc, 4, 2, 64, dtype, 110))


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores_and_scale(dtype):
    """Scores of several hundred: a softmax near one-hot; and a scale of the caller's."""
    pack, enc = wl.make_pack([40], [[9, 9]]), wl.make_enc([150])
    q, k, v, do = _inputs(pack, enc, 4, 2, 64, dtype, 120)
    _check(pack, enc, (q * 16, k, v, do), scale=0.5)
    _check(pack, enc, (q, k, v, do), scale=1e-3)


def test_batches_of_nothing():
    for P, L, E in [([0, 0], [[], []], [3, 0]), ([4], [[2]], [0]), ([0], [[]], [0])]:
        pack, enc = wl.make_pack(P, L), wl.make_enc(E)
        x = [t.to(DEV) for t in _inputs(pack, enc, 4, 2, 64, torch.bfloat16, 130)]
        o, lse = pp.pp_cross_attn_fwd(pack, enc, *x[:3])
        dq, dk, dv = pp.pp_cross_attn_bwd(pack, enc, *x[:3], o, lse, x[3])
        for t in (o, lse, dq, dk, dv):
            assert (t == 0).all()


def test_not_finite_scores_stay_in_their_rows():
    """A NaN query makes its own row NaN; states in the padding are never read (every other test has NaN there)."""
    pack, enc = wl.make_pack([40], [[9, 9]]), wl.make_enc([150])
    for dtype in DTYPES:
        x = _inputs(pack, enc, 4, 2, 64, dtype, 140)
        base = _run(pack, enc, x)
        x[0][7, 2, 5] = float("nan")
        o, lse, dq, _, _ = _run(pack, enc, x)
        bad = torch.zeros(58, 4, dtype=torch.bool, device=DEV)
        bad[7, 2] = True
        assert o[bad].isnan().all() and lse.T[bad].isnan().all() and dq[bad].isnan().all()
        for a, b in ((o, base[0]), (lse.T, base[1].T), (dq, base[2])):
            assert torch.equal(a[~bad], b[~bad])


def test_runs_agree_bit_for_bit():
    pack, enc = wl.make_pack([300, 20], [[100, 50], [3]]), wl.make_enc([1000, 64])
    x = _inputs(pack, enc, 14, 2, 64, torch.bfloat16, 150)
    for a, b in zip(_run(pack, enc, x), _run(pack, enc, x)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("ranges", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_few_keys_keep_the_gradients_digits(hq, hkv, d, ranges):
    """Tokens that see two to four keys, where dP - delta is small beside delta: delta may not carry the
    rounding of the stored O.  With r the error of P (cross_check.py: (d + 4) 2^-24 tau |q| |k| and exp2's and
    lse's few 2^-21, twice) and e = d 2^-24:
      err(delta) <= sum P (2 r |dP| + e |dO| |v|)
      err(dS)    <= |dS| (2^-8 + 2 r) + P (e |dO| |v| + err(delta))
      err(dQ)    <= tau err(dS) |k| + 2^-8 |dQ|, and as much for dK over the rows."""
    n, E = 40, 2.0 ** -24
    pack, enc = wl.make_pack([n, n], [[], []]), wl.make_enc([60, 62] if ranges else [2, 3])
    T = pack.total_tokens
    q, k, v, do = _inputs(pack, enc, hq, hkv, d, torch.bfloat16, 900)
    k *= 3.0  # peaked: most of a row's weight on one key
    rng = np.random.default_rng(3)
    begin = rng.integers(0, 50, T) if ranges else np.zeros(T, int)
    end = begin + rng.integers(2, 5, T) if ranges else np.full(T, 60)
    kw = {}
    if ranges:
        kw = {"key_begin": torch.tensor(begin, dtype=torch.int32, device=DEV), "key_end": torch.tensor(end, dtype=torch.int32, device=DEV)}
    g = [t.to(DEV) for t in (q, k, v, do)]
    o, lse = pp.pp_cross_attn_fwd(pack, enc, *g[:3], **kw)
    dq, dk, _ = (t.double().cpu().numpy() for t in pp.pp_cross_attn_bwd(pack, enc, *g[:3], o, lse, g[3], **kw))
    q, k, v, do = (t.double().numpy() for t in (q, k, v, do))
    tau = 1.0 / np.sqrt(d)
    want_k, tol_k = np.zeros(k.shape), np.zeros(k.shape)
    for t in range(T):
        b = int(t >= n)
        lo, hi = int(begin[t]), min(int(end[t]), int(enc.enc_len[b]))
        keys = slice(int(enc.enc_start[b]) + lo, int(enc.enc_start[b]) + hi)
        for h in range(hq):
            kk, vv, qq, gg = k[keys, h * hkv // hq], v[keys, h * hkv // hq], q[t, h], do[t, h]
            s = tau * kk @ qq
            P = np.exp(s - s.max())
            P /= P.sum()
            dP = vv @ gg
            dS = P * (dP - P @ dP)
            r = 2 * ((d + 4) * E * tau * (np.abs(kk) @ np.abs(qq)) + 4 * E * (np.abs(s) + np.abs(s).max()) + 2.0 ** -21).max()
            fp = d * E * (np.abs(vv) @ np.abs(gg))
            err = np.abs(dS) * (2.0 ** -8 + 2 * r) + P * (fp + (P * (2 * r * np.abs(dP) + fp)).sum())
            ref = tau * dS @ kk
            assert (np.abs(dq[t, h] - ref) <= tau * err @ np.abs(kk) + 2.0 ** -8 * np.abs(ref)).all(), (t, h)
            want_k[keys, h * hkv // hq] += tau * np.outer(dS, qq)
            tol_k[keys, h * hkv // hq] += tau * np.outer(err + T * hq * E * np.abs(dS), np.abs(qq))
    assert (np.abs(dk - want_k) <= tol_k + 2.0 ** -8 * np.abs(want_k)).all()
