"""GPU tests of the attention over the paged cache against the 64-bit oracle, within derived bounds: single tokens and trees,
lengths from none to many, page sizes, pages shared by groups, ragged and padded batches, split walks.

The bounds are cross attention's (cross_check.py): with u the half step of the probabilities' and results' type, e = 2^-24, a
row's greatest score error r = (d + 4) e tau |q|.|k| + 4 e (|s| + |m|) + 2^-21 (|s| and |m| at most tau |q|.|k|) and N keys,
  O    (u + 2 r + 2^-20 + (N + 64) e) P.|v| + u |O|      (2^-20: the exponentials that join partial results)
  lse  r + 2^-20 + (N + 64) e + 4 e |lse|."""
import numpy as np
import pytest
import torch

from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def random_tree(rng, n, width=3):
    return [-1] + [int(rng.integers(max(0, i - width), i)) if rng.random() < 0.9 else -1 for i in range(1, n)]


class Case:
    """Groups of k sequences of which the first `shared` pages are the group's; pages of the others scattered; rows of the
    pools that no sequence has written hold NaN."""

    def __init__(self, dtype, hq, hkv, d, ps, lens, group=1, shared=(), nodes=1, count=None, seed=0, sigma=1.0):
        rng = np.random.default_rng(seed)
        n = len(lens)
        self.dtype, self.group, self.n, self.nodes = dtype, group, n, nodes
        self.count = [nodes] * n if count is None else count
        live = [max(0, min(c, nodes)) for c in self.count]
        held = [-(-(a + c) // ps) for a, c in zip(lens, live)]
        pages = sum(held) + 3
        order = rng.permutation(pages).tolist()
        self.slots = rng.permutation(n + 2)[:n].tolist()
        table = np.full((n + 2, max(held + [1]) + 1), 1 << 30)  # what lies behind the pages held is not looked at
        for i in range(n):
            for c in range(held[i]):
                lead = i - i % group
                share = group > 1 and i != lead and c < shared[i // group]
                table[self.slots[i], c] = table[self.slots[lead], c] if share else order.pop()
        full = np.zeros((2, n + 2))
        full[0, self.slots], full[1, self.slots] = lens, held
        self.cache = pp.Cache(ints(table), ints(full[0]), ints(full[1]), ints(np.zeros(pages)), ps)
        k, v = (wl.randn((pages, hkv, ps, d), seed + 1 + i, dtype, "cpu", sigma=sigma if i == 0 else 1.0) for i in range(2))
        used = np.zeros((pages, ps), bool)
        for i in range(n):
            for t in range(lens[i] + live[i]):
                used[table[self.slots[i], t // ps], t % ps] = True
        for x in (k, v):
            x.transpose(1, 2)[torch.from_numpy(~used)] = float("nan")
        self.k, self.v = k, v
        self.q = wl.randn((n, nodes, hq, d), seed + 3, dtype, "cpu")
        self.shared = ints(shared) if len(shared) else None
        self.parents = [random_tree(rng, nodes) for _ in range(n)]

    def run(self, chains=False, **kw):
        a = self.q.to(DEV)
        ws = torch.full((pp.pp_tree_workspace_size(self.cache, self.n, self.group, self.nodes, a.shape[2], self.k.shape[1],
                                                   a.shape[3], pp._dtype_code(a)),), 0xff, dtype=torch.uint8, device=DEV)
        nan = torch.full_like(a, float("nan"))
        lse = torch.full((a.shape[2], self.n * self.nodes), float("nan"), device=DEV)
        out = pp.pp_tree_attn_fwd(self.cache, ints(self.slots), a, self.k.to(DEV), self.v.to(DEV),
                                  parents=None if chains else ints(self.parents), count=ints(self.count), group=self.group,
                                  shared=self.shared, out=nan, lse=lse, ws=ws, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, chains=False, scale=0.0):
        o, lse = (x.double().cpu().numpy() for x in self.run(chains, scale=scale))
        n64 = lambda t: t.double().numpy()[None]
        tab = self.cache.page_table.cpu().numpy()
        b = smp.Book(tab, self.cache.seq_len.cpu().numpy(), self.cache.held.cpu().numpy(), [], self.cache.page_size, n64(self.k),
                     n64(self.v))
        q, u, d = self.q.double().numpy(), U[self.dtype], self.q.shape[3]
        wo, wl_, size, s = smp.tree_attn(b, 0, self.slots, q, None if chains else self.parents, self.count, scale or None)
        assert (np.isnan(o) == np.isnan(wo)).all() and (np.isnan(lse) == np.isnan(wl_)).all()
        N = int(max(b.len)) + self.nodes
        r = ((d + 4) * E + 8 * E) * s + 2.0 ** -21
        bo = (u + 2 * r + 2.0 ** -20 + (N + 64) * E)[..., None] * size + u * np.abs(wo)
        bl = (r + 2.0 ** -20 + (N + 64) * E).transpose(2, 0, 1).reshape(wl_.shape) + 4 * E * np.abs(wl_)
        ok = ~np.isnan(wo)
        assert (np.abs(o - wo)[ok] <= bo[ok]).all(), float((np.abs(o - wo) - bo)[ok].max())
        ok = ~np.isnan(wl_)
        assert (np.abs(lse - wl_)[ok] <= bl[ok]).all(), float((np.abs(lse - wl_) - bl)[ok].max())
        for i, c in enumerate(self.count):  # nodes not in use
            c = max(0, c)
            assert (o[i, c:] == 0).all() and (lse.reshape(-1, self.n, self.nodes)[:, i, c:] == 0).all()
        return o, lse


HEADS = [(4, 4, 64), (14, 2, 64), (32, 8, 128), (6, 2, 128), (8, 1, 128), (71, 1, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_one_token(dtype, hq, hkv, d):
    Case(dtype, hq, hkv, d, 16, [0, 1, 15, 16, 31, 32, 33, 500], seed=hq).check(chains=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_page_sizes_and_trees(dtype, ps, d):
    Case(dtype, 6, 2, d, ps, [0, 1, ps - 1, ps, ps + 1, 2 * ps + 17, 700], nodes=9, count=[9, 1, 0, 9, 7, 9, 5], seed=ps + d).check()


@pytest.mark.parametrize("nodes", [2, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("chains", [False, True])
def test_tree_sizes(nodes, chains):
    """Masks that begin anywhere in a block of 32 keys and reach over two of its ends."""
    for dtype in (torch.bfloat16, torch.float32):
        Case(dtype, 4, 2, 64, 16, [0, 5, 27, 31, 32, 47, 64], nodes=nodes, seed=nodes).check(chains=chains)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,ps,nodes", [(32, 8, 128, 64, 1), (4, 2, 64, 16, 1), (4, 2, 64, 16, 5), (14, 2, 64, 32, 9),
                                               (8, 1, 128, 16, 20)])
def test_groups(dtype, hq, hkv, d, ps, nodes):
    """Shared pages: none, some, all whole ones; a group with one live sequence, one with none, one with unequal lengths."""
    lens = [5 * ps + 3, 5 * ps + 9, 5 * ps, 3 * ps, 3 * ps, 3 * ps + 1, 7, 8, 9, 2 * ps, 2 * ps, 2 * ps, 4 * ps, 4 * ps, 4 * ps]
    count = [nodes] * 9 + [0, nodes, 0] + [0, 0, 0]
    a = Case(dtype, hq, hkv, d, ps, lens, group=3, shared=[5, 3, 0, 2, 4], nodes=nodes, count=count, seed=nodes)
    o, lse = a.check()
    # the same without the hint: other sums, the same values
    a.shared = None
    o2, lse2 = a.check()
    assert np.nanmax(np.abs(o - o2)) <= 4 * U[dtype] * max(1.0, np.abs(o).max()) and np.nanmax(np.abs(lse - lse2)) <= 1e-4
    # more than the whole pages of the shortest, or less than none
    for pages in (1 << 30, -5):
        a.shared = ints([min(p, pages) if pages < 0 else pages if p * ps == min(lens[3 * i:3 * i + 3]) // ps * ps else p
                         for i, p in enumerate([5, 3, 0, 2, 4])])
        a.check()


def test_split_walks():
    """One sequence over all waves; several that end inside a wave's run; results do not depend on the workspace's contents."""
    for dtype in (torch.bfloat16, torch.float32):
        Case(dtype, 8, 1, 128, 64, [20011], nodes=3, seed=1).check()
        a = Case(dtype, 4, 2, 64, 32, [3000, 1, 777, 9999, 64], nodes=2, seed=2)
        o, lse = a.check()
        o2, lse2 = (x.double().cpu().numpy() for x in a.run())
        np.testing.assert_array_equal(o, o2)
        np.testing.assert_array_equal(lse, lse2)


def test_large_scores():
    """Scores that rise and fall by hundreds: the running maximum is raised late, and never."""
    for dtype in (torch.bfloat16, torch.float32):
        a = Case(dtype, 4, 2, 64, 16, [400, 90, 33], nodes=4, seed=5, sigma=20.0)
        a.check()
        a = Case(dtype, 4, 2, 64, 16, [400, 90, 33], nodes=4, seed=6)
        a.check(scale=3.0)


def test_bad_sequences_and_parents_are_nan():
    a = Case(torch.bfloat16, 4, 2, 64, 16, [20, 33, 40, 16, 5], nodes=5, seed=7)
    a.cache.held[a.slots[1]] -= 1        # the nodes have not all been reserved
    a.cache.seq_len[a.slots[2]] = -1
    a.parents[0] = [-1, 1, 0, 2, 5]      # its own parent; a later one
    a.parents[4] = [-1, 0, -2, 2, 1]
    a.slots[3] = 99
    a.check()
    a.slots[3] = -1                      # left out: zeros
    o, lse = a.run()
    assert (o[3] == 0).all() and (lse.view(4, 5, 5)[:, 3] == 0).all()


def test_pages_that_are_none_are_nan():
    a = Case(torch.float32, 4, 2, 64, 16, [200, 300, 100], nodes=2, seed=8)
    a.cache.page_table[a.slots[1], 7] = 1 << 29
    o, lse = a.run()
    assert torch.isnan(o[1]).all() and torch.isnan(lse.view(4, 3, 2)[:, 1]).all()
    assert torch.isfinite(o[[0, 2]]).all()
    a.cache.page_table[a.slots[1], 7] = -1
    assert torch.isnan(a.run()[0][1]).all()


def test_infinities_and_nan_stay_in_their_sequence():
    a = Case(torch.bfloat16, 4, 2, 64, 16, [200, 300, 100], nodes=2, seed=9)
    page = int(a.cache.page_table[a.slots[1], 3])
    a.k[page, 0, 5, 7], a.v[page, 1, 2, 3] = float("inf"), float("nan")
    o, _ = a.run()
    assert torch.isfinite(o[[0, 2]].float()).all() and not torch.isfinite(o[1].float()).all()


def test_planned_calls_and_streams():
    """A second layer on the first one's plan; another stream; a graph of both, replayed after the cache has grown."""
    a = Case(torch.bfloat16, 4, 2, 64, 16, [100, 7, 64, 65], group=2, shared=[0, 4], nodes=3, seed=10)
    b = Case(torch.bfloat16, 4, 2, 64, 16, [100, 7, 64, 65], group=2, shared=[0, 4], nodes=3, seed=10)
    b.k, b.v, b.q = (x.roll(1, dims=2).contiguous() for x in (b.k, b.v, b.q))
    k, v = (torch.nan_to_num(x).to(DEV) for x in (a.k, a.v))
    k2, v2 = (torch.nan_to_num(x).to(DEV) for x in (b.k, b.v))
    q, q2, slots, par, cnt = a.q.to(DEV), b.q.to(DEV), ints(a.slots), ints(a.parents), ints(a.count)
    kw = dict(parents=par, count=cnt, group=2, shared=a.shared)
    want = pp.pp_tree_attn_fwd(a.cache, slots, q, k, v, **kw), pp.pp_tree_attn_fwd(a.cache, slots, q2, k2, v2, **kw)
    ws = torch.empty(pp.pp_tree_workspace_size(a.cache, 4, 2, 3, 4, 2, 64), dtype=torch.uint8, device=DEV)
    outs = [(torch.empty_like(q), torch.empty(4, 12, device=DEV)) for _ in range(2)]

    def layers():
        pp.pp_tree_attn_fwd(a.cache, slots, q, k, v, ws=ws, out=outs[0][0], lse=outs[0][1], **kw)
        pp.pp_tree_attn_fwd(a.cache, slots, q2, k2, v2, planned=True, ws=ws, out=outs[1][0], lse=outs[1][1], **kw)

    def same(w):
        torch.cuda.synchronize()
        for (o, l), (x, y) in zip(outs, w):
            assert torch.equal(o, x) and torch.equal(l, y)

    layers()
    same(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layers()
    same(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layers()
    for grow in (0, 1, 5, -3):
        a.cache.seq_len += grow
        want = pp.pp_tree_attn_fwd(a.cache, slots, q, k, v, **kw), pp.pp_tree_attn_fwd(a.cache, slots, q2, k2, v2, **kw)
        for o, l in outs:
            o.fill_(7), l.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
        for (o, l), (x, y) in zip(outs, want):
            assert torch.equal(torch.isnan(o), torch.isnan(x)) and torch.equal(bits(torch.nan_to_num(o)), bits(torch.nan_to_num(x)))
            assert torch.equal(bits(torch.nan_to_num(l)), bits(torch.nan_to_num(y)))
    with pytest.raises(ValueError):
        pp.pp_tree_attn_fwd(a.cache, slots, q, k, v, planned=True, **kw)


def test_a_plan_of_another_call_is_refused():
    """planned with a workspace that holds no plan, or one of other sizes: NaN, and nothing is read by it."""
    a = Case(torch.bfloat16, 4, 2, 64, 16, [100, 7, 64, 65], nodes=3, seed=10)
    b = Case(torch.bfloat16, 4, 2, 64, 16, [5, 9], nodes=2, seed=11)
    size = max(pp.pp_tree_workspace_size(a.cache, 4, 1, 3, 4, 2, 64), pp.pp_tree_workspace_size(b.cache, 2, 1, 2, 4, 2, 64))
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    run = lambda x, planned: pp.pp_tree_attn_fwd(x.cache, ints(x.slots), x.q.to(DEV), x.k.to(DEV), x.v.to(DEV), parents=ints(x.parents),
                                                 count=ints(x.count), planned=planned, ws=ws)
    for planned in (lambda: None, lambda: run(b, False)):
        planned()
        o, lse = run(a, True)
        assert torch.isnan(o).all() and torch.isnan(lse).all()
    want = run(a, False)
    assert all(torch.equal(x, y) for x, y in zip(want, run(a, True))) and not torch.isnan(want[0]).any()


@pytest.mark.parametrize("nodes", [3, 40])
def test_numbers_that_are_no_plan(nodes):
    """A workspace of large numbers whose products leave 64 bits, for waves and for teams: NaN."""
    a = Case(torch.bfloat16, 4, 2, 64, 16, [100, 7, 64, 65], nodes=nodes, seed=12)
    ws = torch.zeros(pp.pp_tree_workspace_size(a.cache, 4, 1, nodes, 4, 2, 64) // 8, dtype=torch.int64, device=DEV)
    for x in (0x2000000000000001, 0x7fffffffffffffff, -1):
        ws.fill_(x)
        o, lse = pp.pp_tree_attn_fwd(a.cache, ints(a.slots), a.q.to(DEV), a.k.to(DEV), a.v.to(DEV), planned=True, ws=ws)
        assert torch.isnan(o).all() and torch.isnan(lse).all()


def test_a_pool_past_2_31_elements():
    """Pages whose rows lie past 2^31 elements of the pool."""
    pages, hkv, ps, d = 70000, 2, 256, 64
    k = torch.zeros(pages, hkv, ps, d, dtype=torch.bfloat16, device=DEV)
    assert k.numel() > 2**31
    v = torch.zeros_like(k)
    n = 600
    x = [wl.randn((n, hkv, d), 60 + i, torch.bfloat16, DEV) for i in range(2)]
    order = [pages - 1, 3, pages - 2]
    c = pp.Cache(ints([order]), ints([n - 1]), ints([3]), ints(np.ones(pages)), ps)
    q = wl.randn((1, 1, 4, d), 70, torch.bfloat16, DEV)
    small = pp.Cache(ints([[0, 1, 2]]), ints([n - 1]), ints([3]), ints(np.ones(3)), ps)
    ks, vs = (torch.zeros(3, hkv, ps, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t in range(0, n, ps):
        m = min(ps, n - t)
        for big, little, y in ((k, ks, x[0]), (v, vs, x[1])):
            big[order[t // ps], :, :m] = little[t // ps, :, :m] = y[t:t + m].transpose(0, 1)
    a, b = pp.pp_tree_attn_fwd(c, ints([0]), q, k, v), pp.pp_tree_attn_fwd(small, ints([0]), q, ks, vs)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
