"""CPU tests of cross attention: the oracle against torch's attention and finite differences,
what the library refuses, and the workspace sizes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl


def _case(seed=0):
    rng = np.random.default_rng(seed)
    pack, enc = wl.make_pack([4, 2, 1], [[2, 3], [], [1]], pad=[1, 0, 2]), wl.make_enc([6, 3, 0], pad=[2, 0, 1])
    q = rng.standard_normal((pack.total_tokens, 4, 8))
    k, v = rng.standard_normal((2, enc.total_states, 2, 8))
    return pack, enc, q, k, v, rng.standard_normal(q.shape)


def _ranges(pack):
    begin, end = np.zeros(pack.total_tokens, int), np.full(pack.total_tokens, 9)
    begin[1], end[1] = 2, 5
    begin[2], end[2] = 3, 3  # nothing
    begin[3], end[3] = -4, 100
    begin[5], end[5] = 5, 1  # nothing
    return begin, end


@pytest.mark.parametrize("ranges", [False, True])
def test_oracle_equals_torch_attention(ranges):
    pack, enc, q, k, v, do = _case()
    begin, end = _ranges(pack) if ranges else (None, None)
    o, lse, dq, dk, dv = orc.cross_attn(*pack.oracle_args(), enc.enc_start, enc.enc_len, q, k, v, do, begin, end)
    vis = orc.cross_visible(*pack.oracle_args(), enc.enc_len, begin, end)
    t = [torch.tensor(x, requires_grad=True) for x in (q, k, v)]
    out = torch.zeros(q.shape, dtype=torch.float64)
    parts = []
    for b, see in enumerate(vis):
        rows = int(pack.row_start[b]) + np.nonzero(see.any(axis=1))[0]
        if len(rows) == 0:
            continue
        e = slice(int(enc.enc_start[b]), int(enc.enc_start[b] + enc.enc_len[b]))
        heads = lambda x: x.repeat_interleave(2, dim=1).transpose(0, 1)
        part = torch.nn.functional.scaled_dot_product_attention(
            t[0][rows].transpose(0, 1), heads(t[1][e]), heads(t[2][e]), attn_mask=torch.tensor(see[see.any(axis=1)]))
        out[rows] = part.transpose(0, 1).detach()
        parts.append((part.transpose(0, 1) * torch.tensor(do[rows])).sum())
    sum(parts).backward()
    np.testing.assert_allclose(o, out.numpy(), atol=1e-12)
    for got, want in ((dq, t[0].grad), (dk, t[1].grad), (dv, t[2].grad)):
        np.testing.assert_allclose(got, want.numpy(), atol=1e-12)


def test_oracle_against_differences():
    pack, enc, q, k, v, do = _case(1)
    begin, end = _ranges(pack)
    args = (*pack.oracle_args(), enc.enc_start, enc.enc_len)
    grads = orc.cross_attn(*args, q, k, v, do, begin, end)[2:]
    rng = np.random.default_rng(2)
    for which, g in enumerate(grads):
        x = [q.copy(), k.copy(), v.copy()]
        step = rng.standard_normal(x[which].shape)
        f = []
        for sign in (1, -1):
            y = list(x)
            y[which] = x[which] + sign * 1e-5 * step
            f.append((orc.cross_attn(*args, *y, None, begin, end)[0] * do).sum())
        assert abs((f[0] - f[1]) / 2e-5 - (g * step).sum()) < 1e-8


# ---------------------------------------------------------------- refusals


def _descs(enc_start=(0, 7, 7), enc_len=(5, 0)):
    pack = wl.make_pack([4, 3], [[2], [1]])
    d = pp._DescHolder(pack)
    e = pp._EncHolder(wl.Enc(np.array(enc_start, np.int32), np.array(enc_len, np.int32)))
    return d, e


OK = ctypes.c_void_p(256)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(264)


def _fwd(d, e, dtype=0, hq=4, hkv=2, hd=64, q=OK, k=OK, v=OK, kb=None, ke=None, o=OK, lse=OK, ws=OK, n=1 << 40):
    return pp.lib().pp_cross_attn_fwd(d.ref, e.ref if e else None, dtype, hq, hkv, hd, 0.0, q, k, v, kb, ke, o, lse, ws, n,
                                      None)


def _bwd(d, e, dtype=0, hq=4, hkv=2, hd=64, q=OK, k=OK, v=OK, kb=None, ke=None, o=OK, lse=OK, do=OK, dq=OK, dk=OK, dv=OK,
         ws=OK, n=1 << 40):
    return pp.lib().pp_cross_attn_bwd(d.ref, e.ref if e else None, dtype, hq, hkv, hd, 0.0, q, k, v, kb, ke, o, lse, do, dq, dk,
                                      dv, ws, n, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_bad_arguments_are_refused(call):
    d, e = _descs()
    assert call(d, None) == 1
    assert call(d, e, hq=4, hkv=3) == 1 and call(d, e, dtype=2) == 1
    assert call(d, e, hd=96) == 3 and call(d, e, hq=8192, hkv=1) == 3
    for name in ("q", "k", "v", "o", "lse"):
        assert call(d, e, **{name: None}) == 1, name
    for name in ("q", "k", "v", "o"):
        assert call(d, e, **{name: ODD}) == 1, name
    assert call(d, e, lse=ctypes.c_void_p(258)) == 1
    assert call(d, e, kb=OK) == 1 and call(d, e, ke=OK) == 1 and call(d, e, kb=OK, ke=ctypes.c_void_p(258)) == 1
    if call is _bwd:
        for name in ("do", "dq", "dk", "dv"):
            assert call(d, e, **{name: None}) == 1 and call(d, e, **{name: ODD}) == 1, name
    assert b"16-byte" in pp.lib().pp_last_error() or call is _fwd


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("start,length", [((1, 7, 7), (5, 0)), ((0, 7, 6), (5, 0)), ((0, 4, 7), (5, 0)), ((0, 7, 7), (-1, 0)),
                                          ((0, 7, 7), (5, 1))])
def test_bad_encoder_layouts(call, start, length):
    d, e = _descs(start, length)
    assert call(d, e) == 2


def test_workspaces():
    L = pp.lib()
    pack, enc = wl.make_pack([700], [[300]]), wl.make_enc([3000])
    d, e = pp._DescHolder(pack), pp._EncHolder(enc)
    f, b = pp.pp_cross_workspace_size(pack, enc, 4, 2, 64)
    assert f > 0 and b > 0
    assert _fwd(d, e, n=f - 1) == 4 and _bwd(d, e, n=b - 1) == 4
    assert _fwd(d, e, ws=ODD) == 1 and _bwd(d, e, ws=ODD) == 1 and _fwd(d, e, ws=None) == 1
    assert L.pp_cross_workspace_size(d.ref, e.ref, 0, 4, 2, 64, None, None) == 0
    # the partial sums do not grow with the batch: splitting stops where the tiles fill the card
    for rows in (1, 2, 8, 64):
        many = wl.make_pack([700] * rows, [[300]] * rows), wl.make_enc([3000] * rows)
        f, b = pp.pp_cross_workspace_size(*many, 32, 8, 128)
        assert f <= 80 << 20 and b <= (160 << 20) + 8 * 32 * many[0].total_tokens + (1 << 20)
    # row counts past 31 bits
    huge = wl.Pack(*[np.array(x, np.int32) for x in ([0, 1 << 30], [4], [0])], np.zeros((1, 0), np.int32),
                   np.zeros((1, 0), np.int32))
    assert _fwd(pp._DescHolder(huge), pp._EncHolder(wl.make_enc([4])), hq=4, hkv=1) == 3


def test_the_binding_refuses_what_does_not_fit():
    pack, enc = wl.make_pack([4, 3], [[2], [1]]), wl.make_enc([5, 0], pad=[2, 0])
    q, k = torch.zeros(10, 4, 64), torch.zeros(7, 2, 64)
    with pytest.raises(ValueError):
        pp.pp_cross_attn_fwd(pack, wl.make_enc([5]), q, k, k)
    with pytest.raises(ValueError):
        pp.pp_cross_attn_fwd(pack, enc, q[:9], k, k)
    with pytest.raises(ValueError):
        pp.pp_cross_attn_fwd(pack, enc, q, k[:6], k)
    with pytest.raises(TypeError):
        pp.pp_cross_attn_fwd(pack, enc, q, k.bfloat16(), k)
    with pytest.raises(ValueError):
        pp.pp_cross_attn_fwd(pack, enc, q, torch.zeros(7, 64, 2).transpose(1, 2), k)
    with pytest.raises(TypeError):
        pp.pp_cross_attn_fwd(pack, enc, q, k, k, key_begin=torch.zeros(10), key_end=torch.zeros(10))
    with pytest.raises(ValueError):  # tensors of the host
        pp.pp_cross_attn_fwd(pack, enc, q, k, k)
    with pytest.raises(ValueError):
        wl.make_enc([1 << 30] * 2)
