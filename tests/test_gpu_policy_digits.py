"""GPU tests of the policy loss's digits: terms and sums are 64 bits, so a result is off by
its rounding to fp32 (2^-24 of it) and next to nothing of its parts (2^-40 of their sum of
absolute values: a 64-bit exponential is off by a few 2^-53 and |d| 2^-53, sums of up to
2^11 parts a thread by 2^-42), also where a ratio or e^x of the KL term is past fp32."""
import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E, F = 2.0 ** -24, 2.0 ** -40


def _packs():
    rng = np.random.default_rng(2)
    return {"small": wl.make_pack([20, 3], [[200, 77, 1], [0, 512]], pad=[0, 5]),
            "inline": wl.make_pack([700, 5], [[3000, 900], [2000, 1]]),
            "many": wl.make_pack([300] * 100, [rng.integers(1, 60, size=4).tolist() for _ in range(100)]),
            "wide": wl.make_pack([2900] * 92, [rng.integers(1, 60, size=4).tolist() for _ in range(92)])}


PACKS = _packs()
assert PACKS["small"].total_tokens <= 4096 < PACKS["inline"].total_tokens and PACKS["wide"].total_tokens > 1 << 18


def _check(pack, lp, adv, kw, **cfg):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    names = {"old": "logp_old", "ref": "logp_ref", "entropy": "entropy", "mask": "mask"}
    got = pp.pp_policy_loss(pack, dev(lp), dev(adv), **{names[k]: dev(v) for k, v in kw.items()}, **cfg)
    loss, stats, counts, dlogp, _ = orc.policy_loss(*pack.oracle_args(), lp, adv, **kw, **cfg)
    assert got[2].tolist() == counts.tolist()
    toks = [(t, b, k) for _, t, b, k in orc.response_tokens(*pack.oracle_args()) if kw.get("mask") is None or kw["mask"][t]]
    per = {}
    for _, b, k in toks:
        per[b, k] = per.get((b, k), 0) + 1
    parts, p_lp, c = np.zeros(4), np.zeros(len(lp)), abs(cfg.get("kl_coef", 0.0))
    for t, b, k in toks:
        w = {"token": 1 / len(toks), "seq": 1 / (len(per) * per[b, k]), "sum": 1 / cfg.get("norm", 1.0)}[cfg.get("reduction", "token")]
        A = abs(float(adv[t] if adv.ndim == 1 else adv[b, k]))
        r = np.exp(float(lp[t]) - float(kw["old"][t])) if kw.get("old") is not None else 1.0
        div = dd = 0.0
        if kw.get("ref") is not None:
            x = float(kw["ref"][t]) - float(lp[t])
            div, dd = {"k1": (abs(x), 1.0), "k2": (x * x / 2, abs(x)), "k3": (np.expm1(x) - x, abs(np.expm1(x)))}[cfg.get("kl", "k3")]
        parts += w * np.array([A * max(r, 2.0), div, 0.0, r])
        p_lp[t] = w * (A * r + c * dd)
    if kw.get("entropy") is not None:
        parts[2] = abs(stats[2])
    total = parts[0] + c * parts[1] + abs(cfg.get("ent_coef", 0.0)) * parts[2]
    back = lambda t: t.double().cpu().numpy()
    assert abs(float(got[0]) - loss) <= E * abs(loss) + F * total
    assert (np.abs(back(got[1]) - stats) <= E * np.abs(stats) + F * parts).all(), (got[1], stats)
    assert (np.abs(back(got[3]) - dlogp) <= E * np.abs(dlogp) + F * p_lp + 1e-44).all()
    return got


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("name", sorted(PACKS))
def test_results_are_off_by_their_rounding(name, masked, kl):
    pack = PACKS[name]
    rng = np.random.default_rng(5)
    T, f = pack.total_tokens, lambda a: a.astype(np.float32)
    lp = f(-3 * np.abs(rng.standard_normal(T)))
    kw = {"old": f(lp + 0.3 * rng.standard_normal(T)), "ref": f(lp + rng.choice([1e-5, 1e-2, 0.5, 4.0], T) * rng.standard_normal(T)),
          "entropy": f(rng.random(T)), "mask": rng.random(T) > 0.3 if masked else None}
    adv = f(rng.standard_normal((pack.num_rows, pack.max_resp)))
    for reduction, dual in (("token", 0.0), ("seq", 1.3), ("sum", 2.0)):
        _check(pack, lp, adv, kw, kl_coef=0.3, kl=kl, ent_coef=0.02, reduction=reduction, norm=1000.0, clip_low=0.1, dual_clip=dual)


@pytest.mark.parametrize("name", sorted(PACKS))
@pytest.mark.parametrize("d", [88.0, 89.5, 95.0, 100.0])
def test_ratios_past_fp32(name, d):
    """Negative advantages without a dual clip leave the ratio as it is: where weight and advantage are small, its product
    with them has an fp32 value; so has the mean ratio of tokens without an advantage."""
    pack = PACKS[name]
    T = pack.total_tokens
    rng = np.random.default_rng(6)
    lp = (-rng.random(T)).astype(np.float32)
    old = lp.copy()
    toks = [t for _, t, _, _ in orc.response_tokens(*pack.oracle_args())]
    old[toks[3]] -= np.float32(d)
    old[toks[-2]] -= np.float32(d - 1)
    for size in (-1e-6, 0.0):
        adv = np.full((pack.num_rows, pack.max_resp), size, np.float32)
        got = _check(pack, lp, adv, {"old": old}, reduction="sum", norm=1e7)
        assert got[1].isfinite().all() and got[3].isfinite().all() and float(got[1][3]) > 1e29


@pytest.mark.parametrize("name", sorted(PACKS))
def test_divergences_past_fp32(name):
    pack = PACKS[name]
    T = pack.total_tokens
    rng = np.random.default_rng(7)
    lp = (-rng.random(T)).astype(np.float32)
    ref = lp.copy()
    toks = [t for _, t, _, _ in orc.response_tokens(*pack.oracle_args())]
    ref[toks[5]] += np.float32(91.0)
    ref[toks[6]] -= np.float32(91.0)
    got = _check(pack, lp, np.full((pack.num_rows, pack.max_resp), 0.5, np.float32), {"ref": ref}, kl_coef=1e-3, reduction="sum",
                 norm=1e5)
    assert got[0].isfinite() and got[1].isfinite().all() and got[3].isfinite().all()


def test_log_probs_of_minus_infinity_and_nan():
    """A token that the policy rules out has ratio 0; one that the sampling policy ruled out an infinite one; NaN stays."""
    pack = wl.make_pack([2], [[6]])
    lp, old = torch.full((8,), -1.0, device=DEV), torch.full((8,), -1.0, device=DEV)
    lp[3], old[4], old[5] = float("-inf"), float("-inf"), float("nan")
    adv = torch.full((8,), -1.0, device=DEV)
    *_, dlogp, _ = pp.pp_policy_loss(pack, lp, adv, logp_old=old, reduction="sum")
    assert dlogp[[2, 6, 7]].tolist() == [1.0] * 3 and dlogp[3] == 0 and dlogp[4] == float("inf") and dlogp[5].isnan()
