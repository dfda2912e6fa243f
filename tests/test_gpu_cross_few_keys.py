"""GPU tests of cross attention's gradients where a token sees few keys, wherever they lie:
in any tile of 64 keys, across the border of two, and on both sides of a split axis.
dP - delta is small beside delta there, so delta may not carry the rounding of the stored
O.  With E = 2^-24, r the error of P ((d + 4) E tau |q| |k|, exp2's and lse's few 2^-21, twice;
see cross_check.py) and e = d E:
  err(delta) <= sum P (2 r |dP| + e |dO| |v|)
  err(dS)    <= |dS| (2^-8 + 2 r) + P (e |dO| |v| + err(delta))
  err(dQ)    <= tau err(dS) |k| + 2^-8 |dQ|, and as much for dK over the rows."""
import numpy as np
import pytest
import torch

from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV, BF = "cuda:0", torch.bfloat16
E = 2.0 ** -24


def _check(pack, enc, hq, hkv, d, begin, end, seed, most=64):
    """begin, end per token; tokens that see up to `most` keys are held to the bounds, and dK where only such ones look."""
    T, S = pack.total_tokens, enc.total_states
    q, k, v, do = (wl.randn(s, seed + i, BF, "cpu") for i, s in enumerate([(T, hq, d), (S, hkv, d), (S, hkv, d), (T, hq, d)]))
    k *= 3.0  # peaked: most of a row's weight on one key
    kw = {n: torch.tensor(a, dtype=torch.int32, device=DEV) for n, a in (("key_begin", begin), ("key_end", end))}
    g = [t.to(DEV) for t in (q, k, v, do)]
    o, lse = pp.pp_cross_attn_fwd(pack, enc, *g[:3], **kw)
    dq, dk, _ = (t.double().cpu().numpy() for t in pp.pp_cross_attn_bwd(pack, enc, *g[:3], o, lse, g[3], **kw))
    q, k, v, do = (t.double().numpy() for t in (q, k, v, do))
    tau = 1.0 / np.sqrt(d)
    want_k, tol_k, held = np.zeros(k.shape), np.zeros(k.shape), np.ones(S, bool)
    for b in range(pack.num_rows):
        e0, n = int(enc.enc_start[b]), int(enc.enc_len[b])
        real = int(pack.row_start[b]) + int(pack.prompt_len[b]) + int(pack.resp_len[b, :pack.num_resp[b]].sum())
        for t in range(int(pack.row_start[b]), int(pack.row_start[b + 1])):
            lo, hi = max(0, int(begin[t])), min(int(end[t]), n) if t < real else 0  # padding sees nothing
            if hi <= lo:
                assert (dq[t] == 0).all()
                continue
            keys = slice(e0 + lo, e0 + hi)
            if hi - lo > most:
                held[keys] = False
                continue
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
                assert (np.abs(dq[t, h] - ref) <= tau * err @ np.abs(kk) + 2.0 ** -8 * np.abs(ref)).all(), (t, h, lo, hi)
                want_k[keys, h * hkv // hq] += tau * np.outer(dS, qq)
                tol_k[keys, h * hkv // hq] += tau * np.outer(err + T * hq * E * np.abs(dS), np.abs(qq))
    bad = np.abs(dk - want_k) > tol_k + 2.0 ** -8 * np.abs(want_k)
    assert not bad[held].any(), np.argwhere(bad & held[:, None, None])[:5]


HEADS = [(8, 2, 128), (6, 2, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_ranges_anywhere(hq, hkv, d):
    n = 60
    pack, enc = wl.make_pack([n, n], [[], []]), wl.make_enc([200, 333])
    rng = np.random.default_rng(4)
    begin = rng.integers(0, 196, 2 * n)
    _check(pack, enc, hq, hkv, d, begin, begin + rng.integers(1, 5, 2 * n), 910)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_ranges_across_tile_borders(hq, hkv, d):
    n = 48
    pack, enc = wl.make_pack([n, n], [[], []]), wl.make_enc([200, 129])
    rng = np.random.default_rng(5)
    size = rng.integers(2, 6, 2 * n)
    border = 64 * np.concatenate([rng.integers(1, 4, n), rng.integers(1, 3, n)])
    begin = border - 1 - rng.integers(0, 4, 2 * n) % np.maximum(size - 1, 1)
    _check(pack, enc, hq, hkv, d, begin, begin + size, 920)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_images_of_up_to_one_tile_at_odd_places(hq, hkv, d):
    """Images of 1 to 64 states one after the other: a token sees the one ahead of it, and later ones in between see all."""
    rng = np.random.default_rng(6)
    sizes = [64, 3, 64, 17, 50, 64, 1, 2, 40]
    at = np.cumsum([0] + sizes)
    pack, enc = wl.make_pack([90], [[30, 7]], pad=[3]), wl.make_enc([int(at[-1])], pad=[5])
    T = pack.total_tokens
    which = np.sort(rng.integers(0, len(sizes), T))
    begin, end = at[which], at[which + 1]
    _check(pack, enc, hq, hkv, d, begin, end, 930)
    begin, end = begin.copy(), end.copy()
    begin[::9], end[::9] = 0, 2 ** 31 - 1
    begin[4::9], end[4::9] = end[4::9], begin[4::9]  # sees nothing
    _check(pack, enc, hq, hkv, d, begin, end, 940)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_ranges_across_parts_of_a_split_axis(hq, hkv, d):
    """Few tokens and many states: the keys of a row tile are walked by several workgroups."""
    n, S = 20, 4000
    pack, enc = wl.make_pack([n, 3], [[], []]), wl.make_enc([S, 700])
    fwd, bwd = pp.pp_cross_workspace_size(pack, enc, hq, hkv, d)
    rng = np.random.default_rng(7)
    border = 64 * np.concatenate([rng.permutation(np.arange(1, S // 64))[:n], rng.integers(1, 10, 3)])
    for size in (2, 3, 64, 63):
        begin = border - rng.integers(1, size, n + 3)
        _check(pack, enc, hq, hkv, d, begin, begin + size, 950 + size)
        begin[::2], end = 0, begin + size
        end[::2] = S
        _check(pack, enc, hq, hkv, d, begin, end, 960 + size)
