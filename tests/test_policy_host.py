"""CPU tests of the policy-optimisation oracles (finite differences, torch, closed forms) and
of what the library refuses."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

PACK = wl.make_pack([4, 2, 1], [[2, 3], [], [1, 0, 5]], pad=[1, 0, 2])
ARGS = PACK.oracle_args()
T = PACK.total_tokens


def test_tok_logprob_oracle():
    rng = np.random.default_rng(0)
    x, y = 2 * rng.standard_normal((T, 11)), rng.integers(0, 11, T)
    x[:, 9] = -np.inf
    y[y == 9] = 0
    tok, ent = orc.tok_logprob(*ARGS, x, y)
    seq, per = orc.seq_logprob(*ARGS, x, y)
    np.testing.assert_allclose(tok, per, atol=1e-13)
    lp = torch.log_softmax(torch.tensor(x), 1)
    H = torch.special.entr(lp.exp()).sum(1).numpy()
    for r, t, _, _ in orc.response_tokens(*ARGS):
        assert abs(ent[t] - H[r]) < 1e-13
    dtok, dent = rng.standard_normal((2, T))
    g = orc.tok_logprob_grad(*ARGS, x, y, dtok, dent)
    assert (g[:, 9] == 0).all()
    step = rng.standard_normal(x.shape)
    f = [sum((a * b).sum() for a, b in zip(orc.tok_logprob(*ARGS, np.where(np.isinf(x), x, x + h * step), y), (dtok, dent)))
         for h in (1e-6, -1e-6)]
    assert abs((f[0] - f[1]) / 2e-6 - (g * np.where(np.isinf(x), 0, step)).sum()) < 1e-7


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("reduction", ["token", "seq", "sum"])
@pytest.mark.parametrize("dual", [0.0, 2.0])
def test_policy_oracle_against_differences(kl, reduction, dual):
    rng = np.random.default_rng(1)
    lp, ent, adv = -rng.random(T), rng.random(T), rng.standard_normal((3, 3))
    kw = dict(old=lp + 0.8 * rng.standard_normal(T), ref=lp + 0.3 * rng.standard_normal(T), mask=rng.random(T) > 0.3,
              dual_clip=dual, kl_coef=0.1, kl=kl, ent_coef=0.05, reduction=reduction, norm=7.0)
    loss, stats, counts, dlogp, dent = orc.policy_loss(*ARGS, lp, adv, entropy=ent, **kw)
    assert counts[1] > 0 and loss == pytest.approx(stats[0] + 0.1 * stats[1] - 0.05 * stats[2], abs=1e-14)
    s1, s2 = rng.standard_normal((2, T))
    f = [orc.policy_loss(*ARGS, lp + h * s1, adv, entropy=ent + h * s2, **kw)[0] for h in (1e-7, -1e-7)]
    assert abs((f[0] - f[1]) / 2e-7 - (dlogp * s1 + dent * s2).sum()) < 1e-6


def test_policy_oracle_closed_forms():
    lp, adv = -np.ones(T), np.ones((3, 3))
    loss, stats, counts, dlogp, _ = orc.policy_loss(*ARGS, lp, adv)  # on-policy: ratio 1
    assert loss == pytest.approx(-1) and counts.tolist() == [11, 0] and stats[3] == pytest.approx(1)
    assert dlogp.sum() == pytest.approx(-1)
    up = orc.policy_loss(*ARGS, lp + 1, adv, old=lp)  # every ratio e: clipped
    assert up[0] == pytest.approx(-1.2) and up[2][1] == 11 and (up[3] == 0).all()
    down = orc.policy_loss(*ARGS, lp + 1, -adv, old=lp)  # a negative advantage is not clipped there
    assert down[0] == pytest.approx(np.e) and down[2][1] == 0
    dual = orc.policy_loss(*ARGS, lp + 1, -adv, old=lp, dual_clip=2.0)
    assert dual[0] == pytest.approx(2) and dual[2][1] == 11 and (dual[3] == 0).all()
    none = orc.policy_loss(*ARGS, lp, adv, mask=np.zeros(T))
    assert none[0] == 0 and none[2].tolist() == [0, 0]


# ---------------------------------------------------------------- refusals

OK, ODD = ctypes.c_void_p(256), ctypes.c_void_p(258)


def _desc(pack=PACK):
    return pp._DescHolder(pack)


def _policy(d=None, cfg=None, logp=OK, old=None, ref=None, ent=None, adv=OK, mask=None, loss=OK, stats=None, counts=None,
            dlogp=None, dent=None, ws=OK, n=1 << 30, **c):
    vals = dict(clip_low=0.2, clip_high=0.2, dual_clip=0.0, kl_coef=0.0, ent_coef=0.0, norm=1.0, kl=2, reduction=0)
    vals.update(c)
    cfg = pp._PolicyConfig(**vals) if cfg is None else cfg
    return pp.lib().pp_policy_loss((d or _desc()).ref, ctypes.byref(cfg), logp, old, ref, ent, adv, 0, mask, loss, stats, counts,
                                   dlogp, dent, ws, n, None)


def test_policy_refusals():
    assert pp.lib().pp_policy_loss(_desc().ref, None, OK, None, None, None, OK, 0, None, OK, None, None, None, None, OK, 1 << 30,
                                   None) == 1
    for bad in ({"clip_low": -0.1}, {"clip_low": 1.5}, {"clip_low": float("nan")}, {"clip_high": -1.0},
                {"clip_high": float("inf")}, {"dual_clip": 1.0}, {"dual_clip": float("nan")}, {"kl_coef": float("inf")},
                {"ent_coef": float("nan")}, {"kl": 3}, {"kl": -1}, {"reduction": 3}, {"reduction": 2, "norm": 0.0},
                {"reduction": 2, "norm": float("nan")}, {"kl_coef": 0.1}, {"ent_coef": 0.1}, {"dent": OK}, {"loss": None},
                {"logp": None}, {"adv": None}, {"logp": ODD}, {"old": ODD}, {"dlogp": ODD}, {"ws": OK.value + 16}):
        assert _policy(**bad) == 1, bad
        assert pp.lib().pp_last_error()
    # a few tokens of few responses need no workspace; others do
    assert pp.pp_policy_workspace_size(PACK) == 0
    for big in (wl.make_pack([20000], [[5]]), wl.make_pack([1], [[1] * 300])):
        assert pp.pp_policy_workspace_size(big) > 0
        assert _policy(_desc(big), n=1) == 4 and _policy(_desc(big), ws=None) == 1
    assert pp.lib().pp_policy_workspace_size(_desc().ref, None) == 1


def test_tok_logprob_refusals():
    L, d = pp.lib(), _desc()
    n = 1 << 30
    no_prompt = _desc(wl.make_pack([0], [[5]]))
    assert L.pp_tok_logprob(no_prompt.ref, 0, 10, OK, OK, OK, None, OK, n, None) == 2
    assert L.pp_tok_logprob(d.ref, 0, 0, OK, OK, OK, None, OK, n, None) == 1
    assert L.pp_tok_logprob(d.ref, 5, 10, OK, OK, OK, None, OK, n, None) == 1
    for i in range(3):
        p = [OK, OK, OK]
        p[i] = None
        assert L.pp_tok_logprob(d.ref, 0, 10, *p, None, OK, n, None) == 1
    assert L.pp_tok_logprob(d.ref, 0, 10, OK, OK, OK, None, OK, 1, None) == 4
    assert L.pp_tok_logprob(d.ref, 0, 10, OK, OK, OK, None, ODD, n, None) == 1
    many = _desc(wl.make_pack([3], [[1] * 257]))
    for call in (lambda h, *a: L.pp_tok_logprob_bwd(h.ref, *a),
                 lambda h, dt, V, x, y, g, e, out, *rest: L.pp_tok_logprob_bwd_rows(h.ref, dt, V, x, y, g, e, out, None, *rest)):
        assert call(no_prompt, 0, 10, OK, OK, OK, None, OK, OK, n, None) == 2
        assert call(many, 0, 10, OK, OK, OK, None, OK, OK, n, None) == 3
        for i in (0, 1, 2, 4):
            p = [OK, OK, OK, None, OK]
            p[i] = None
            assert call(d, 0, 10, *p, OK, n, None) == 1
        assert call(d, 0, 10, OK, OK, OK, None, OK, OK, 1, None) == 4


def test_the_binding_refuses_what_does_not_fit():
    x, y, f = torch.zeros(T, 7), torch.zeros(T, dtype=torch.int32), torch.zeros(T)
    for bad in ((x[:-1], y), (x, y[:-1]), (x[0], y), (x.t().contiguous().t(), y)):
        with pytest.raises(ValueError):
            pp.pp_tok_logprob(PACK, *bad)
    with pytest.raises(TypeError):
        pp.pp_tok_logprob(PACK, x, y.long())
    with pytest.raises(TypeError):
        pp.pp_tok_logprob(PACK, x.half(), y)
    with pytest.raises(ValueError):
        pp.pp_tok_logprob_bwd(PACK, x, y, f[:-1])
    adv = torch.zeros(3, 3)
    for kw in ({"adv": adv[:2]}, {"adv": f[1:]}, {"logp_old": f[1:]}, {"kl": "k4"}, {"reduction": "mean"}, {}):
        with pytest.raises(ValueError):  # the last: tensors of the host
            pp.pp_policy_loss(PACK, f, **{"adv": adv, **kw})
    with pytest.raises(TypeError):
        pp.pp_policy_loss(PACK, f, adv, mask=f)
