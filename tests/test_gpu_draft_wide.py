"""GPU tests of draft verification where rows have more than 64 and 128 stretches of 2048 entries, which other parts of the
kernels join and search: just below, at and above both, with what decides lying in any of them; and logits past 2^31 elements.
Equality and tolerances as in test_gpu_draft.py."""
import numpy as np
import pytest
import torch

from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl
from test_gpu_draft import DEV, DTYPES, case, check, ints

pytestmark = pytest.mark.gpu

WIDE = [131072 - 7, 131073, 262144 - 7, 262144, 270001]
TOP_U = 1 - 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", WIDE)
def test_plain_sampling(dtype, V):
    """A flat distribution: the numbers decide the stretch, the first and the last of them too."""
    u = np.array([0.0, TOP_U, 0.25, 0.49, 0.51, 0.97, 0.99, 0.999, 0.9999], np.float32)[:, None]
    target = wl.randn((len(u), 1, V), V, dtype, "cpu", sigma=0.5)
    out = check(target, np.zeros((len(u), 1), int), u, temperature=[1.0] * 6 + [0.0, 2.0, 1.0])
    assert out[1][0, 0] < 2048 and out[1][1, 0] >= V - 2048 and out[1][5, 0] // 2048 > 60


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", WIDE)
def test_rejected_siblings(dtype, V):
    """Sums of what is left after one to three children, and the next token out of them."""
    target, tokens, u, draft, _ = case(6, 4, V, dtype, V % 1000, near=4.0, sigma=1.0)
    u[:, 1:] = np.maximum(u[:, 1:], 0.9)
    u[:, 0] = [0.0, TOP_U, 0.3, 0.6, 0.9, 0.99]
    again = tokens.copy()
    again[:, 2:] = tokens[:, 1:2]  # nothing is left of a token that was rejected
    for kids, toks in ((1, tokens), (3, tokens), (3, again)):
        for d in (draft, None):
            out = check(target, toks, u, d, [[-1, 0, 0, 0]] * 6, max_children=kids)
            assert (out[0] == 1).any() or toks is tokens and kids == 3


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("stretch", [0, 63, 64, 127, 128, 131])
def test_given_drafts_that_are_all_of_a_stretch(dtype, stretch):
    """Rejected drafts hold (all but) all of one stretch; the smallest number finds what is left there, or behind it, or, from
    the last one, ahead of it."""
    rng, n, V = np.random.default_rng(stretch), 24, 270001
    first, behind = 2048 * stretch + 20, 2048 * (stretch + 2) if stretch < 128 else 2048 * 5
    for faint in (False, True):
        target = torch.full((n, 4, V), -float("inf"), dtype=dtype)
        target[:, :, behind:behind + 50] = torch.tensor(rng.normal(0, 1, (n, 4, 50)), dtype=dtype)
        tokens = np.zeros((n, 4), int)
        for i in range(n):
            tokens[i, 1:] = first + rng.choice(1000, size=3, replace=False)
            target[i, :, torch.tensor(tokens[i, 1:])] = torch.tensor(rng.normal(2.5, 1, 3), dtype=dtype)
        if faint:
            target[:, :, first + 1200] = -46.0
        u = np.full((n, 4), 0.9995, np.float32)
        u[:, 0] = 0
        count, out, _, _ = check(target, tokens, u, None, [[-1, 0, 0, 0]] * n, max_children=3)
        assert (count == 1).all() and (out[:, 0] == (first + 1200 if faint and behind > first else behind)).all()
        u[:, 0] = TOP_U
        check(target, tokens, u, None, [[-1, 0, 0, 0]] * n, max_children=3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_decides_lies_far_behind(dtype):
    """Maxima, masks, NaN and +inf in stretches 64 and up, 128 and up; also greedy and cold."""
    V, at = 270001, [2048 * 64 + 1, 2048 * 127 + 2047, 2048 * 128, 270000]
    target, tokens, u, draft, _ = case(14, 3, V, dtype, 9, width=1, sigma=1.0)
    low = torch.finfo(dtype).min
    for i, y in enumerate(at):
        target[i, :, y] = 9.0
        draft[i, :, y] = 9.0
        tokens[i, 1:] = y
        target[4 + i, 0, y] = float("nan")
        draft[8 + i, 1, y] = float("inf") if i % 2 else float("nan")
    target[12, :, :at[2]] = low
    draft[12, :, :at[2]] = low
    tokens[12, 1:] = 269000
    target[13, :, 100:] = -float("inf")
    tokens[13, 1:] = 200000
    for temp in (None, [0.0] * 14, [0.05] * 14):
        for d in (draft, None):
            out = check(target, tokens, u, d, temperature=temp)
            if temp and temp[0] == 0:
                assert (out[1][:4, 0] == at).all() and (out[0][:4] == 3).all()
            assert (out[1][4:8, 0] == -1).all() and np.isnan(out[3][4:8, 0]).all()


def test_logits_past_2_31_elements():
    """Sequences whose rows lie past 2^31 elements of the model's and the drafter's logits."""
    n, N, V = 2051, 4, 262144
    assert n * N * V > 2**31
    live = [0, 1023, n - 2, n - 1]
    t = torch.zeros(n, N, V, dtype=torch.bfloat16, device=DEV)
    d = torch.zeros_like(t)
    target, tokens, u, draft, parents = case(len(live), N, V, torch.bfloat16, 13, near=2.0)
    t[live], d[live] = target.to(DEV), draft.to(DEV)
    count, all_tokens, all_u, par = np.zeros(n, int), np.zeros((n, N), int), np.zeros((n, N), np.float32), np.full((n, N), -1)
    count[live], all_tokens[live], all_u[live], par[live] = N, tokens, u, parents
    for dd, draft_ in ((d, draft), (None, None)):
        got = pp.pp_verify_draft(t, ints(all_tokens), torch.tensor(all_u, device=DEV), dd, ints(par), ints(count), max_children=2)
        want = smp.verify(target.double().numpy(), tokens, u.astype(np.float64), None if draft_ is None else draft_.double().numpy(), parents,
                          max_children=2)
        for g, w in zip(got[:3], want):
            np.testing.assert_array_equal(g[live].cpu().numpy(), w)
        lp, w = got[3][live].double().cpu().numpy(), want[3]
        assert (np.abs(lp - w) <= 2.0 ** -24 * np.abs(w) + 1e-12).all()
        rest = np.setdiff1d(np.arange(n), live)
        assert (got[0].cpu().numpy()[rest] == 0).all() and (got[1].cpu().numpy()[rest] == -1).all()


@pytest.mark.parametrize("drafted", [True, False])
def test_all_children_of_a_tree_by_default(drafted):
    target, tokens, u, draft, _ = case(40, 5, 500, torch.bfloat16, 77, drafted, near=4.0)
    args = target.to(DEV), ints(tokens), torch.tensor(u, device=DEV), None if draft is None else draft.to(DEV), ints([[-1, 0, 0, 0, 0]] * 40)
    got, want = pp.pp_verify_draft(*args), pp.pp_verify_draft(*args, max_children=4)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not drafted or (got[2][:, 1] > 1).any()  # a later child follows


@pytest.mark.parametrize("drafted", [True, False])
def test_nodes_whose_parent_is_no_earlier_one(drafted):
    """They are never reached, nor what hangs from them; the others are as they would be without."""
    target, tokens, u, draft, _ = case(30, 6, 60, torch.float32, 31, drafted, near=0.3)
    u[:, 1:] = 0.01
    for parents in ([-1, 0, 4, 2, 0, 3], [-1, 1, 0, 0, 9, 2], [5, 0, 1, -7, 3, 2**31 - 1], [-1, -1, 0, 3, 2, 4]):
        out = check(target, tokens, u, draft, [parents] * 30, max_children=5)
        kept = set(out[2].ravel().tolist()) - {-1}
        reach = {0}
        for j in range(1, 6):
            if 0 <= parents[j] < j and parents[j] in reach:
                reach.add(j)
        assert kept <= reach and (not drafted or len(kept) > 1)
