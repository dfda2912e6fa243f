"""GPU tests of the token log-probs with entropies, their gradient, and the clipped policy
loss against the 64-bit oracle.

Tolerances, with E = 2^-24.  The kernels sum a row's exponentials in fp32, a thread every
1024th vector, so a sum passes C = V / 1024 + 64 roundings at most (V where a row is that
short).  With X the greatest |logit - row maximum| that has weight (a masked entry has
none) plus the greatest such |logit|, an exponent is off by 2 E X log2(e) and the hardware's exp2
by 2^-22:
  log-prob   E (4 X + C + 64) + 4 E |lp|
  entropy    E (4 X + C + 64) (1 + sum p |x - m|) + 4 E H
  dlogits    p (|c| + |h| (|ln p| + H)) E (8 X + 2 C + 128) + |h| p err(H)
             + 2^-126 (|c| + |h| (|ln p| + H)): the hardware's exp2 gives 0 for what lies
             below fp32's normal range, an error of p of less than 2^-126
             + E 300 sum |g| at labels, plus half a step of the output's type
             (bf16 2^-8 |v|, fp32 2^-24 |v|)
The loss's terms are fp32, its sums 64 bits.  With d = logp - old and x = ref - logp, each
rounded once (E |d|, E |x|):
  r = e^d        r E (4 + 2 |d|)                       (expf: one step, and d's rounding)
  surrogate      |A| r E (8 + 2 |d|)
  KL             k1 E |x|;  k2 4 E x^2 / 2;
                 k3 and its derivative e^x - 1: |x| <= 1/2 a series of 9 terms, each no larger than a sixth of
                 the one before: 12 E of the value; else 6 E (|e^x - 1| + |x|) + E |x| e^x
  gradient       w (the surrogate's and |kl_coef| times the derivative's errors) + 4 E of both parts
which outputs counts is decided exactly."""
import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
# every form a row can take: single elements, registers of each shape, off the boundaries, streamed
SHAPES = [(1, F32), (5, F32), (9, BF), (200, BF), (4096, F32), (4099, BF), (20003, F32), (50257, BF), (77831, F32), (131072, F32),
          (152064, BF), (155661, BF), (163840, BF)]


def _pack():
    return wl.make_pack([3, 1, 2], [[4, 2], [1, 0, 3], []], pad=[1, 0, 2])


def _check_tok(pack, x, y, dtok, dent):
    V, args = x.shape[1], pack.oracle_args()
    xg, yg, tg = x.to(DEV), y.to(DEV), dtok.to(DEV)
    eg = None if dent is None else dent.to(DEV)
    tok, ent = pp.pp_tok_logprob(pack, xg, yg, want_entropy=True)
    plain, none = pp.pp_tok_logprob(pack, xg, yg)
    assert none is None
    dl = pp.pp_tok_logprob_bwd(pack, xg, yg, tg, eg)
    dr, ri = pp.pp_tok_logprob_bwd_rows(pack, xg, yg, tg, eg)
    assert torch.equal(dr.view(torch.uint8), dl[ri.long()].view(torch.uint8))
    off = torch.ones(len(dl), dtype=torch.bool, device=DEV)
    off[ri.long()] = False
    assert (dl[off] == 0).all()
    xn, yn = x.double().numpy(), y.numpy()
    gn, hn = dtok.double().numpy(), np.zeros(len(y)) if dent is None else dent.double().numpy()
    want_tok, want_ent = orc.tok_logprob(*args, xn, yn)
    want_dl = orc.tok_logprob_grad(*args, xn, yn, gn, hn)
    tok, plain, ent, dl = (t.double().cpu().numpy() for t in (tok, plain, ent, dl))
    C = (V / 1024 if V > 4096 else V) + 64
    seen = np.zeros(len(y), bool)
    rows = {}
    for r, t, _, _ in orc.response_tokens(*args):
        rows.setdefault(r, []).append(t)
        seen[t] = True
    assert (tok[~seen] == 0).all() and (ent[~seen] == 0).all() and (plain[~seen] == 0).all()
    u = 2.0 ** -8 if x.dtype == BF else E
    for r, ts in rows.items():
        p, lp = orc._row_softmax(xn[r])
        real = p > 0  # a masked entry has no weight
        m = xn[r].max()
        X = np.abs(xn[r][real] - m).max() + (np.abs(xn[r][real]).max() if abs(m) < 1e30 else 0.0)
        spread = (p[real] * np.abs(xn[r][real] - m)).sum()
        H = -(p[real] * lp[real]).sum()
        err_h = E * (4 * X + C + 64) * (1 + spread) + 4 * E * H
        for t in ts:
            for got in (tok[t], plain[t]):
                if abs(want_tok[t]) < 1e30:
                    far = abs(xn[r][yn[t]] - m) + X
                    assert abs(got - want_tok[t]) <= E * (4 * far + C + 64) + 4 * E * abs(want_tok[t]), (r, t)
                else:
                    assert got == pytest.approx(want_tok[t], rel=1e-6)
            assert abs(ent[t] - want_ent[t]) <= err_h, (r, t, ent[t], want_ent[t])
        c, h = sum(abs(gn[t]) for t in ts), sum(abs(hn[t]) for t in ts)
        size = np.where(p > 0, np.abs(np.where(p > 0, lp, 0.0)), 0.0)
        bar = (p * E * (8 * X + 2 * C + 128) + 2.0 ** -126 * (p > 0)) * (c + h * (size + H)) + h * p * err_h
        for t in ts:
            bar[yn[t]] += E * 300 * c
        bar += u * (np.abs(want_dl[r]) + bar) + 1e-38
        assert (np.abs(dl[r] - want_dl[r]) <= bar).all(), (r, (np.abs(dl[r] - want_dl[r]) / bar).max())


def _inputs(V, dtype, seed, sigma=3.0):
    pack = _pack()
    T = pack.total_tokens
    return (pack, wl.randn((T, V), seed, dtype, "cpu", sigma=sigma), wl.randint((T,), V, seed + 1, "cpu"),
            wl.randn((T,), seed + 2, F32, "cpu"), wl.randn((T,), seed + 3, F32, "cpu"))


@pytest.mark.parametrize("V,dtype", SHAPES)
def test_tok_logprob(V, dtype):
    pack, x, y, g, h = _inputs(V, dtype, 500)
    _check_tok(pack, x, y, g, h)
    _check_tok(pack, x, y, g, None)


@pytest.mark.parametrize("kind", ["neginf", "lowest", "lowest_row", "peak", "flat", "large"])
@pytest.mark.parametrize("V,dtype", [(9, BF), (4096, F32), (4099, BF), (131072, F32), (163840, BF)])
def test_tok_logprob_extremes(V, dtype, kind):
    pack, x, y, g, h = _inputs(V, dtype, 520)
    lo, hi = V // 3, max(V // 3 + 1, V // 2)
    if kind in ("neginf", "lowest"):
        y = lo + y % (hi - lo)
        value = -float("inf") if kind == "neginf" else torch.finfo(dtype).min
        x[:, :lo], x[:, hi:] = value, value
    elif kind == "lowest_row":
        x[:] = torch.finfo(dtype).min
    elif kind == "peak":  # one entry holds almost all: the entropy nears 0
        x[:, lo] = 60.0
    elif kind == "flat":
        x[:] = 0.25
    else:
        x *= 300
    _check_tok(pack, x, y, g, h)


def test_tok_logprob_not_finite_and_bad_labels():
    for V, dtype in [(200, F32), (4099, BF), (163840, BF)]:
        pack, x, y, g, h = _inputs(V, dtype, 540)
        ref = [t.clone() for t in pp.pp_tok_logprob(pack, x.to(DEV), y.to(DEV), want_entropy=True)]
        dref = pp.pp_tok_logprob_bwd(pack, x.to(DEV), y.to(DEV), g.to(DEV), h.to(DEV))
        # rows of pack: 2 predicts positions 3 and 7; 3 predicts 4; a label of position 5 is bad (row 4)
        x[3, V // 2] = float("nan")
        y[5] = V
        x[0, 0] = float("nan")  # predicts nothing
        tok, ent = pp.pp_tok_logprob(pack, x.to(DEV), y.to(DEV), want_entropy=True)
        dl = pp.pp_tok_logprob_bwd(pack, x.to(DEV), y.to(DEV), g.to(DEV), h.to(DEV))
        assert tok[4].isnan() and ent[4].isnan() and tok[5].isnan() and ent[5] == ref[1][5]
        same = torch.ones(len(y), dtype=torch.bool, device=DEV)
        same[[4, 5]] = False
        assert torch.equal(tok[same], ref[0][same]) and torch.equal(ent[same], ref[1][same])
        assert dl[3].isnan().all() and dl[4].isnan().all()
        same[[3, 4, 5]] = torch.tensor([False, False, True], device=DEV)
        assert torch.equal(dl[same], dref[same])


def test_tok_logprob_agrees_with_the_sequence_form():
    """Without entropies and with a response's weight on all its tokens, bit for bit."""
    pack, x, y, _, _ = _inputs(50257, BF, 560)
    xg, yg = x.to(DEV), y.to(DEV)
    dseq = wl.randn((pack.num_rows, pack.max_resp), 561, F32, "cpu")
    dtok = torch.full((pack.total_tokens,), float("nan"))
    for _, t, b, k in orc.response_tokens(*pack.oracle_args()):
        dtok[t] = dseq[b, k]
    _, per = pp.pp_seq_logprob(pack, xg, yg, want_tok=True)
    assert torch.equal(pp.pp_tok_logprob(pack, xg, yg)[0], per)
    assert torch.equal(pp.pp_tok_logprob_bwd(pack, xg, yg, dtok.to(DEV)), pp.pp_seq_logprob_bwd(pack, xg, yg, dseq.to(DEV)))


# ---------------------------------------------------------------- the loss


def _policy_case(pack, seed, adv_tok=False, old=True, ref=True, entropy=True, masked=True):
    rng = np.random.default_rng(seed)
    T, f = pack.total_tokens, lambda a: a.astype(np.float32)
    lp = f(-np.abs(rng.standard_normal(T)))
    kw = {"old": f(lp + 0.4 * rng.standard_normal(T)) if old else None,
          "ref": f(lp + 0.3 * rng.standard_normal(T)) if ref else None,
          "entropy": f(rng.random(T)) if entropy else None, "mask": rng.random(T) > 0.2 if masked else None}
    adv = f(rng.standard_normal(T if adv_tok else (pack.num_rows, max(1, pack.max_resp))))
    # what is not counted holds no number
    counted = np.zeros(T, bool)
    for _, t, _, _ in orc.response_tokens(*pack.oracle_args()):
        counted[t] = kw["mask"] is None or kw["mask"][t]
    for a in (lp, kw["old"], kw["ref"], kw["entropy"], adv if adv_tok else None):
        if a is not None:
            a[~counted] = np.nan
    return lp, adv, kw


def _check_policy(pack, lp, adv, kw, at=0, **cfg):
    """at: elements by which the per-token arrays are off an allocation's start."""
    def dev(a):
        if a is None:
            return None
        t = torch.from_numpy(np.ascontiguousarray(a))
        if t.dim() != 1 or t.dtype == torch.bool:
            return t.to(DEV)
        return torch.cat([torch.zeros(at), t]).to(DEV)[at:]
    names = {"old": "logp_old", "ref": "logp_ref", "entropy": "entropy", "mask": "mask"}
    ws = torch.full((max(1, pp.pp_policy_workspace_size(pack)),), 0xff, dtype=torch.uint8, device=DEV)
    got = pp.pp_policy_loss(pack, dev(lp), dev(adv), **{names[k]: dev(v) for k, v in kw.items()}, ws=ws, **cfg)
    loss, stats, counts, dlogp, dent = orc.policy_loss(*pack.oracle_args(), lp, adv, **kw, **cfg)
    back = lambda t: t.double().cpu().numpy()
    assert got[2].tolist() == counts.tolist()
    # every counted token's allowance, in 64 bits
    toks = [(t, b, k) for _, t, b, k in orc.response_tokens(*pack.oracle_args()) if kw.get("mask") is None or kw["mask"][t]]
    per = {}
    for _, b, k in toks:
        per[b, k] = per.get((b, k), 0) + 1
    b_lp, b_sum = np.zeros(len(lp)), np.zeros(4)
    red, c = cfg.get("reduction", "token"), abs(cfg.get("kl_coef", 0.0))
    for t, b, k in toks:
        w = {"token": 1 / len(toks), "seq": 1 / (len(per) * per[b, k]), "sum": 1 / cfg.get("norm", 1.0)}[red]
        A = abs(float(adv[t] if adv.ndim == 1 else adv[b, k]))
        d = abs(float(lp[t]) - float(kw["old"][t])) if kw.get("old") is not None else 0.0
        r = np.exp(float(lp[t]) - float(kw["old"][t])) if kw.get("old") is not None else 1.0
        e_kl = e_d = size = 0.0
        if kw.get("ref") is not None:
            x = float(kw["ref"][t]) - float(lp[t])
            em = np.expm1(x)
            e_kl, e_d, size = {"k1": (abs(x), 0.0, 1.0), "k2": (2 * x * x, abs(x), abs(x)),
                               "k3": (12 * (em - x), 12 * abs(em), abs(em)) if abs(x) <= 0.5 else
                               (6 * (abs(em) + abs(x)) + abs(x) * np.exp(x),) * 2 + (abs(em),)}[cfg.get("kl", "k3")]
        b_lp[t] = E * w * (A * r * (12 + 2 * d) + c * (e_d + 4 * size))
        b_sum += E * w * np.array([A * r * (8 + 2 * d), e_kl, 0.0, r * (4 + 2 * d)])
    b_loss = b_sum[0] + c * b_sum[1]
    back = lambda t: t.double().cpu().numpy()
    assert abs(float(got[0]) - loss) <= b_loss * 1.001 + E * abs(loss) + 1e-12
    assert (np.abs(back(got[1]) - stats) <= b_sum * 1.001 + E * np.abs(stats) + 1e-12).all()
    assert (np.abs(back(got[3]) - dlogp) <= b_lp * 1.001 + 1e-44).all()
    if got[4] is not None:
        assert (np.abs(back(got[4]) - dent) <= E * np.abs(dent) * (1 + 1e-6) + 1e-44).all()
    return got


@pytest.mark.parametrize("reduction", ["token", "seq", "sum"])
@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
def test_policy_loss(reduction, kl):
    pack = wl.make_pack([5, 1, 3, 0], [[300, 7], [1, 0, 64, 255], [], []], pad=[3, 0, 9, 4])
    for seed, (tok, old, ref, ent, masked) in enumerate([(0, 1, 1, 1, 1), (1, 1, 1, 0, 0), (0, 0, 1, 1, 0), (1, 1, 0, 0, 1)]):
        lp, adv, kw = _policy_case(pack, seed, tok, old, ref, ent, masked)
        _check_policy(pack, lp, adv, kw, clip_low=0.2, clip_high=0.28, dual_clip=[0.0, 1.5][seed % 2],
                      kl_coef=0.05 if ref else 0.0, kl=kl, ent_coef=0.01 if ent else 0.0, reduction=reduction, norm=37.0)


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("masked", [False, True])
def test_policy_past_one_workgroup(masked, kl):
    """More tokens than one workgroup takes, of few responses."""
    pack = wl.make_pack([9000, 300], [[700, 2000, 5], [6000, 1]], pad=[0, 40])
    assert pack.total_tokens > 4096
    lp, adv, kw = _policy_case(pack, 11, True, masked=masked)
    for reduction in ("token", "seq", "sum"):
        _check_policy(pack, lp, adv, kw, kl_coef=0.2, kl=kl, ent_coef=0.01, reduction=reduction, norm=99.0)


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("masked", [False, True])
def test_policy_many_responses(masked, at):
    """More responses than the launch's arguments hold; more tokens than one pass of single tokens takes; odd alignment."""
    rng = np.random.default_rng(7)
    pack = wl.make_pack(rng.integers(1, 3000, size=150).tolist(), [rng.integers(0, 400, size=5).tolist() for _ in range(150)],
                        pad=rng.integers(0, 900, size=150).tolist())
    assert pack.total_tokens > 1 << 18
    lp, adv, kw = _policy_case(pack, 3, True, masked=masked)
    for reduction in ("token", "seq"):
        _check_policy(pack, lp, adv, kw, at=at, kl_coef=0.1, ent_coef=0.01, reduction=reduction)


def test_policy_responses_of_one_token():
    pack = wl.make_pack([1] * 40, [[1] * 12] * 40)
    for masked in (False, True):
        lp, adv, kw = _policy_case(pack, 5, masked=masked)
        for reduction in ("token", "seq"):
            _check_policy(pack, lp, adv, kw, kl_coef=0.1, reduction=reduction)


def test_policy_borders_of_the_clip():
    """Ratios next to the clip's ends, and exact ones."""
    pack = wl.make_pack([1], [[64]])
    T = pack.total_tokens
    for low, high, dual in [(0.2, 0.28, 3.0), (1.0, 0.0, 0.0), (0.0, 0.0, 1.25)]:
        ends = [np.log1p(high), np.log1p(-low) if low < 1 else -80.0, np.log(dual) if dual else 1.0, 0.0]
        old = np.zeros(T, np.float32)
        lp = np.concatenate([np.float32(ends), np.nextafter(np.float32(ends), np.float32(9)),
                             np.nextafter(np.float32(ends), np.float32(-9))] * 6).astype(np.float32)[:T]
        lp = np.concatenate([lp, np.zeros(max(0, T - len(lp)), np.float32)])
        for sign in (1, -1, 0):
            adv = np.full((1, 1), sign, np.float32)
            _check_policy(pack, lp, adv, {"old": old}, clip_low=low, clip_high=high, dual_clip=dual)


def test_policy_nothing_counted():
    for pack in (wl.make_pack([4], [[]], max_resp=2), wl.make_pack([0], [[]]), wl.make_pack([3], [[2, 1]])):
        T = pack.total_tokens
        z, adv = torch.full((T,), float("nan"), device=DEV), torch.full((1, max(1, pack.max_resp)), float("nan"), device=DEV)
        mask = torch.zeros(T, dtype=torch.uint8, device=DEV)
        for reduction in ("token", "seq", "sum"):
            loss, stats, counts, dlogp, dent = pp.pp_policy_loss(pack, z, adv, logp_old=z, logp_ref=z, entropy=z, mask=mask,
                                                                 kl_coef=0.1, ent_coef=0.1, reduction=reduction)
            for t in (loss, stats, counts, dlogp, dent):
                assert (t == 0).all()


def test_policy_small_divergence_keeps_its_digits():
    """e^x - 1 - x of x near 1e-4: a difference of nearly equal numbers in fp32."""
    pack = wl.make_pack([1], [[100]])
    rng = np.random.default_rng(0)
    lp = (-rng.random(101)).astype(np.float32)
    ref = (lp + 1e-4 * rng.standard_normal(101)).astype(np.float32)
    got = _check_policy(pack, lp, np.zeros((1, 1), np.float32), {"ref": ref}, kl_coef=1.0)
    want = orc.policy_loss(*pack.oracle_args(), lp, np.zeros((1, 1)), ref=ref, kl_coef=1.0)[1][1]
    assert float(got[1][1]) == pytest.approx(want, rel=12 * E + E)


@pytest.mark.parametrize("lens", [[3, 2], [3000, 2]])
def test_policy_ratio_past_fp32_without_advantage(lens):
    pack = wl.make_pack([4], [lens])
    T = pack.total_tokens
    lp, old = torch.full((T,), -1.0, device=DEV), torch.full((T,), -1.0, device=DEV)
    old[5] = -101.0  # e^100 is past fp32, its product with an advantage of 0 is 0
    loss, stats, counts, dlogp, _ = pp.pp_policy_loss(pack, lp, torch.tensor([[0.0, 1.0]], device=DEV), logp_old=old, reduction="sum")
    assert loss.item() == -2.0 and stats[0].item() == -2.0 and counts.tolist() == [sum(lens), 0]
    want = torch.zeros(T, device=DEV)
    want[4 + lens[0]:] = -1.0
    assert torch.equal(dlogp, want)
