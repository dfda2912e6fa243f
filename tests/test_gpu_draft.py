"""GPU tests of draft verification against the oracle: whole numbers equal, log-probs within their rounding; chains and trees,
siblings, given drafts, greedy sequences, masks, rows that cannot be used, vocabularies that end anywhere.

Numbers u are fp32 and probabilities 64 bits on both sides, whose sums differ by some 1e-14 of the whole: that one of a few
thousand comparisons falls in between has a chance below 1e-9.  A log-prob is ln p rounded to fp32: 2^-24 |ln p| + 1e-12."""
import numpy as np
import pytest
import torch

from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPES = [torch.bfloat16, torch.float32]


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def case(n, N, V, dtype, seed, drafted=True, width=2, near=0.7, sigma=2.0):
    rng = np.random.default_rng(seed)
    target = wl.randn((n, N, V), seed, dtype, "cpu", sigma=sigma)
    draft = (target.float() + near * wl.randn((n, N, V), seed + 1, torch.float32, "cpu")).to(dtype) if drafted else None
    parents = [[-1] + [int(rng.integers(max(0, i - width), i)) for i in range(1, N)] for _ in range(n)]
    src = (draft if drafted else target).double()
    tokens = np.zeros((n, N), int)
    for i in range(n):
        for j in range(1, N):
            p = torch.softmax(src[i, parents[i][j]], 0).numpy()
            tokens[i, j] = rng.choice(V, p=p / p.sum())
    return target, tokens, rng.random((n, N)).astype(np.float32), draft, parents


def check(target, tokens, u, draft=None, parents=None, count=None, temperature=None, max_children=1):
    n, N, V = target.shape
    opt = lambda x, f: None if x is None else f(x)
    ws = torch.full((pp.pp_verify_workspace_size(n, N, V, pp._dtype_code(target)),), 0xff, dtype=torch.uint8, device=DEV)
    got = pp.pp_verify_draft(target.to(DEV), ints(tokens), torch.tensor(u, device=DEV), opt(draft, lambda t: t.to(DEV)),
                             opt(parents, ints), opt(count, ints), opt(temperature, lambda t: torch.tensor(t, dtype=torch.float32, device=DEV)),
                             max_children, ws=ws)
    torch.cuda.synchronize()
    low = -3.38e38 if target.dtype == torch.bfloat16 else -3.4e38
    want = smp.verify(target.double().numpy(), tokens, u.astype(np.float64), opt(draft, lambda t: t.double().numpy()), parents, count,
                      opt(temperature, lambda t: np.asarray(t, np.float32)), max_children, low)
    for name, g, w in zip(("count", "tokens", "path"), got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)
    g, w = got[3].double().cpu().numpy(), want[3]
    assert (np.isnan(g) == np.isnan(w)).all()
    assert (np.abs(np.nan_to_num(g) - np.nan_to_num(w)) <= 2.0 ** -24 * np.abs(np.nan_to_num(w)) + 1e-12).all()
    return want


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 255, 1000, 8191, 8192, 8193, 20011])
def test_plain_sampling(dtype, V):
    """One node a sequence: the first entry at which the running sum passes u, also for u = 0 and the largest u below 1."""
    target, tokens, u, _, _ = case(9, 1, V, dtype, V, drafted=False)
    u[0], u[1], u[2] = 0.0, 1 - 2.0 ** -24, 0.5
    check(target, tokens, u, temperature=[1.0, 1.0, 0.0, 0.5, 3.0, 1.0, -1.0, float("nan"), 1.0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("N,V,kids", [(2, 50, 1), (5, 1001, 1), (9, 300, 3), (24, 9000, 2), (64, 130, 4)])
def test_trees(dtype, drafted, N, V, kids):
    rng = np.random.default_rng(N)
    for seed in range(3):
        target, tokens, u, draft, parents = case(12, N, V, dtype, 100 * seed + N, drafted, width=kids + 1)
        out = check(target, tokens, u, draft, parents, count=rng.integers(0, N + 2, size=12).tolist(),
                    temperature=rng.choice([1.0, 0.6, 1.5, 0.0], size=12).tolist(), max_children=kids)
        assert not drafted or out[0].max() > 1  # something is kept (given drafts: with p(y), test_given_drafts_of_a_sharp_model)


@pytest.mark.parametrize("dtype", DTYPES)
def test_given_drafts_of_a_sharp_model(dtype):
    target, tokens, u, _, parents = case(20, 12, 4000, dtype, 91, False, sigma=12.0)
    out = check(target, tokens, u, None, parents, max_children=2)
    assert out[0].max() > 3


def test_rejections_go_through_every_sibling():
    """A draft far from the model: most children are rejected, and what is left is sampled from after one to four of them."""
    for drafted in (True, False):
        for dtype in DTYPES:
            target, tokens, u, draft, _ = case(40, 5, 500, dtype, 77, drafted, near=4.0)
            parents = [[-1, 0, 0, 0, 0]] * 40
            for kids in (1, 2, 4, 64):
                out = check(target, tokens, u, draft, parents, max_children=kids)
            assert (out[0] == 1).any() and (out[0] > 1).any()


def test_chains_without_parents():
    target, tokens, u, draft, _ = case(16, 6, 777, torch.bfloat16, 5, width=1)
    check(target, tokens, u, draft)
    check(target, tokens, u, None)


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_same_token_twice_among_siblings(dtype):
    target, tokens, u, draft, _ = case(30, 5, 40, dtype, 11, near=2.0)
    tokens[:, 2] = tokens[:, 1]
    tokens[:, 4] = tokens[:, 1]
    u[:, 1] = 0.999
    parents = [[-1, 0, 0, 0, 0]] * 30
    check(target, tokens, u, draft, parents, max_children=4)
    check(target, tokens, u, None, parents, max_children=4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("faint", [False, True])
def test_given_drafts_that_are_all_of_a_stretch(dtype, faint):
    """The rejected drafts hold all, or all but 10^-20, of the vocabulary's first entries: the smallest u still finds an entry
    that is left, the faint one or else the first behind them."""
    rng, n, V = np.random.default_rng(5), 96, 9000
    target = torch.full((n, 4, V), -float("inf"), dtype=dtype)
    target[:, :, 6000:6050] = torch.tensor(rng.normal(0, 1, (n, 4, 50)), dtype=dtype)
    tokens = np.zeros((n, 4), int)
    for i in range(n):
        tokens[i, 1:] = rng.choice(np.arange(10, 1500), size=3, replace=False)
        target[i, :, torch.tensor(tokens[i, 1:])] = torch.tensor(rng.normal(2.5, 1, 3), dtype=dtype)
    if faint:
        target[:, :, 1700] = -46.0
    u = np.full((n, 4), 0.9995, np.float32)
    u[:, 0] = 0
    count, out, _, _ = check(target, tokens, u, None, [[-1, 0, 0, 0]] * n, max_children=3)
    assert (count == 1).all() and (out[:, 0] == (1700 if faint else 6000)).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_and_rows_that_cannot_be_used(dtype):
    target, tokens, u, draft, _ = case(14, 3, 9000, dtype, 21, width=1)
    low = torch.finfo(dtype).min
    target[0, :, 4000:] = -np.inf
    target[1, :, :8990] = low
    draft[1, :, :8990] = low
    tokens[1, 1:] = 8995
    target[2, 0, 5] = np.nan
    target[3, 0, 8999] = np.inf
    target[4, 0, :] = -np.inf
    target[5, 1, :] = low
    draft[6, 0, 17] = np.nan
    draft[7, 0, :] = -np.inf
    draft[8, 1, 3] = np.inf
    tokens[9, 1], tokens[10, 1] = -1, 9000
    draft[11, 0, int(tokens[11, 1])] = -np.inf  # a token that the drafter could not have drawn
    target[12, 0, int(tokens[12, 1])] = -np.inf
    target[13, 0, :] = low
    target[13, 0, 8500] = 3.0
    for temp in (None, [0.0] * 14, [0.3] * 14):
        check(target, tokens, u, draft, temperature=temp)
        check(target, tokens, u, None, temperature=temp)


@pytest.mark.parametrize("dtype", DTYPES)
def test_nan_anywhere_in_a_row(dtype):
    """A NaN beside ordinary logits, among masked ones, among logits far below the largest; also at low temperatures."""
    target, tokens, u, draft, _ = case(10, 2, 9001, dtype, 27, width=1)
    low = torch.finfo(dtype).min
    for i, (node, at, around) in enumerate([(0, 0, None), (0, 9000, None), (0, 5000, -np.inf), (0, 5000, low), (1, 3000, -np.inf),
                                            (0, 5000, float("nan")), (0, 5000, -3e4), (1, 8999, -3e4)]):
        for x in (target, draft) if i % 2 else (target,):
            if around is not None:
                x[i, node, 2048 * (at // 2048):2048 * (at // 2048) + 2048] = around
            x[i, node, at] = float("nan")
    draft[8, 0, 77] = float("nan")
    for temp in (None, [0.01] * 10, [0.0] * 10):
        for d in (draft, None):
            out = check(target, tokens, u, d, temperature=temp)
    assert np.isnan(out[3]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [0.0, 300.0])
def test_hot_and_cold(dtype, offset):
    """Temperatures from the smallest number to the largest that is told apart, also far from zero."""
    temps = [1e-45, 1e-38, 1e-20, 1e-9, 1e-6, 1e-4, 1e-3, 0.01, 0.1, 10.0, 1e3, 1e5, 1e6]
    target, tokens, u, draft, parents = case(len(temps), 4, 5000, dtype, 41, near=0.3)
    target, draft = ((x.float() + offset).to(dtype) for x in (target, draft))
    check(target, tokens, u, draft, parents, temperature=temps, max_children=2)
    check(target, tokens, u, None, parents, temperature=temps, max_children=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [-300.0, -12.0, 12.0])
def test_logits_of_one_sign(dtype, offset):
    """Rows whose entries are all negative (as log-probs are) or all positive, stretches of them among others, masks beside
    them, zeros of both signs as the largest, NaN with a sign."""
    target, tokens, u, draft, parents = case(9, 4, 7001, dtype, 43, near=0.3)
    target, draft = ((x.float() + offset).to(dtype) for x in (target, draft))
    for x in (target, draft):
        x[1, :, 2000:5000] = -float("inf")
        x[2, :, 4096:6144] = torch.finfo(dtype).min
        x[3, :, 2048:4096] -= 2 * offset  # a stretch of the other sign
    for i, zeros in ((4, (-0.0, 0.0)), (5, (0.0, -0.0)), (6, (-0.0, -0.0))):
        target[i] = -target[i].abs() - 1
        target[i, :, 1111], target[i, :, 6666] = zeros
    sign = torch.tensor(-1, dtype=torch.int16 if dtype == torch.bfloat16 else torch.int32).view(dtype)  # a NaN
    target[7, 0, 4321] = sign
    draft[8, 0, 6999] = sign
    assert torch.isnan(target[7, 0, 4321]) and torch.isnan(draft[8, 0, 6999])
    for temp in (None, [0.7] * 9, [0.0] * 9):
        for d in (draft, None):
            out = check(target, tokens, u, d, parents, temperature=temp, max_children=2)
    assert [out[1][i, out[0][i] - 1] for i in (4, 5, 6)] == [1111] * 3 and np.isnan(out[3][7]).any()


def test_greedy_takes_the_first_largest():
    target, tokens, u, draft, _ = case(6, 4, 20000, torch.bfloat16, 31, width=1)
    for i in range(6):
        for a in range(4):
            target[i, a, [19000 - a, 70 + i, 8192 * 2 - 1]] = 30.0
            if a < 3:
                tokens[i, a + 1] = 70 + i if i % 2 else 19000 - a
    out = check(target, tokens, u, draft, temperature=[0.0] * 6)
    assert out[0].tolist() == [1, 4, 1, 4, 1, 4] and (out[1][np.arange(6), out[0] - 1] == 70 + np.arange(6)).all()


def test_rows_off_the_16_byte_boundaries():
    """Tensors that start anywhere, target and draft differently; odd vocabularies."""
    for dtype, V in ((torch.bfloat16, 9001), (torch.float32, 8203)):
        target, tokens, u, draft, parents = case(6, 4, V, dtype, 41, near=2.0)
        for a, b in ((1, 0), (0, 3), (1, 1), (3, 2)):
            t, d = (torch.empty(x.numel() + 8, dtype=dtype, device=DEV)[o:o + x.numel()].view(x.shape) for x, o in ((target, a), (draft, b)))
            t.copy_(target), d.copy_(draft)
            got = pp.pp_verify_draft(t, ints(tokens), torch.tensor(u, device=DEV), d, ints(parents), max_children=2)
            want = smp.verify(target.double().numpy(), tokens, u.astype(np.float64), draft.double().numpy(), parents, max_children=2)
            for g, w in zip(got[:3], want):
                np.testing.assert_array_equal(g.cpu().numpy(), w)


def test_large_vocabulary_many_numbers():
    """A flat distribution over 152064 entries: 64-bit sums decide where u passes."""
    rng = np.random.default_rng(2)
    target = wl.randn((64, 1, 152064), 51, torch.bfloat16, "cpu", sigma=0.5)
    check(target, np.zeros((64, 1), int), rng.random((64, 1)).astype(np.float32))


def test_distribution_of_what_comes_out():
    """20000 sequences of one distribution with drafts drawn from another: the first new tokens' counts against p, each within
    five standard deviations."""
    rng = np.random.default_rng(8)
    V, n = 12, 20000
    p_row, q_row = rng.standard_normal((2, V)) * 1.2
    soft = lambda x: np.exp(x) / np.exp(x).sum()
    p, q = soft(p_row.astype(np.float32).astype(float)), soft(q_row.astype(np.float32).astype(float))
    N = 3
    target = torch.tensor(p_row, dtype=torch.float32).expand(n, N, V).contiguous().to(DEV)
    draft = torch.tensor(q_row, dtype=torch.float32).expand(n, N, V).contiguous().to(DEV)
    tokens = np.zeros((n, N), int)
    tokens[:, 1:] = rng.choice(V, p=q, size=(n, N - 1))
    u = torch.tensor(rng.random((n, N)).astype(np.float32), device=DEV)
    par = ints(np.tile([-1, 0, 0], (n, 1)))
    _, out, _, _ = pp.pp_verify_draft(target, ints(tokens), u, draft, par, max_children=2)
    got = np.bincount(out[:, 0].cpu().numpy(), minlength=V)
    assert (np.abs(got - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_stream_and_graph():
    target, tokens, u, draft, parents = case(8, 6, 3000, torch.bfloat16, 61, near=1.5)
    t, d, tok, par = target.to(DEV), draft.to(DEV), ints(tokens), ints(parents)
    uu = torch.tensor(u, device=DEV)
    f = lambda: pp.pp_verify_draft(t, tok, uu, d, par, max_children=2)
    want = f()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = f()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = f()
    for seed in range(4):
        uu.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(seed)))
        want = f()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_binding_refuses():
    target, tokens, u, draft, parents = case(2, 3, 50, torch.float32, 71)
    t, tok, uu = target.to(DEV), ints(tokens), torch.tensor(u, device=DEV)
    for bad in (lambda: pp.pp_verify_draft(t[0], tok, uu), lambda: pp.pp_verify_draft(t, tok.long(), uu),
                lambda: pp.pp_verify_draft(t, tok, uu.double()), lambda: pp.pp_verify_draft(t, tok[:, :2], uu),
                lambda: pp.pp_verify_draft(t, tok, uu, t.bfloat16()), lambda: pp.pp_verify_draft(t[:, :, ::2], tok, uu),
                lambda: pp.pp_verify_draft(t, tok, uu, count=ints([1])), lambda: pp.pp_verify_draft(t.cpu(), tok, uu)):
        with pytest.raises((ValueError, TypeError)):
            bad()
