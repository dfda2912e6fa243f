"""GPU tests of the attention over the paged cache where workers walk far: many blocks of keys through their rings, several
items in one run, more pages than a wave holds numbers of, maxima that rise from block to block.  Compared on the GPU with 64-bit
products over each sequence's pages, within test_gpu_tree.py's bounds; each case says, from the plan in the workspace, how many
units its workers take."""
import numpy as np
import pytest
import torch

from paper_2602_24082_amd import binding as pp
from test_gpu_tree import DEV, E, U, ints, random_tree

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


class Walk:
    """Sequences of given lengths on scattered pages, each group's first `shared` ones its own; rows that no sequence has
    written hold NaN."""

    def __init__(self, dtype, hq, hkv, d, ps, lens, nodes=1, group=1, shared=None, count=None, seed=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        n = len(lens)
        self.dtype, self.heads, self.lens, self.nodes, self.group = dtype, (hq, hkv, d), lens, nodes, group
        self.count = [nodes] * n if count is None else count
        held = [-(-(a + c) // ps) for a, c in zip(lens, self.count)]
        order = rng.permutation(sum(held) + 3).tolist()
        table = np.full((n, max(held) + 1), 1 << 30)
        for i in range(n):
            lead = i - i % group
            for c in range(held[i]):
                share = shared is not None and i != lead and c < shared[i // group]
                table[i, c] = table[lead, c] if share else order.pop()
        randn = lambda *shape: torch.randn(shape, generator=g, device=DEV).to(dtype)
        self.k, self.v = randn(sum(held) + 3, hkv, ps, d), randn(sum(held) + 3, hkv, ps, d)
        for i in range(n):
            tail = (lens[i] + self.count[i]) % ps
            if tail:
                for x in (self.k, self.v):
                    x[int(table[i, held[i] - 1]), :, tail:] = float("nan")
        self.q = randn(n, nodes, hq, d)
        self.table = torch.tensor(table, device=DEV)
        self.cache = pp.Cache(self.table.int(), ints(lens), ints(held), ints(np.zeros(sum(held) + 3)), ps)
        self.parents = [random_tree(rng, nodes) for _ in range(n)]
        self.shared = None if shared is None else ints(shared)

    def pages(self, i):
        ps = self.cache.page_size
        return self.table[i, :-(-(self.lens[i] + self.count[i]) // ps)]

    def check(self):
        """Runs and compares; units in all and of a worker, of those that waves take and of the teams'."""
        hq, hkv, d = self.heads
        n, N, G, u = len(self.lens), self.nodes, hq // hkv, U[self.dtype]
        ws = torch.full((pp.pp_tree_workspace_size(self.cache, n, self.group, N, hq, hkv, d, pp._dtype_code(self.q)),), 0xff,
                        dtype=torch.uint8, device=DEV)
        o, lse = pp.pp_tree_attn_fwd(self.cache, ints(np.arange(n)), self.q, self.k, self.v, parents=ints(self.parents),
                                     count=ints(self.count), group=self.group, shared=self.shared, ws=ws)
        for i in range(n):
            c, L = self.count[i], self.lens[i]
            if c == 0:
                assert (o[i] == 0).all()
                continue
            of = lambda pool: pool[self.pages(i)].double().transpose(0, 1).reshape(hkv, -1, d)[:, :L + c].contiguous()
            k, v = of(self.k), of(self.v)
            q = self.q[i, :c].double().view(c, hkv, G, d).transpose(0, 1).reshape(hkv, c * G, d) * d ** -0.5
            see = torch.zeros(c, c, dtype=torch.bool)
            for j in range(c):
                up = self.parents[i][j]
                if up >= 0:
                    see[j] = see[up]
                see[j, j] = True
            hide = torch.zeros(c * G, L + c, dtype=torch.bool, device=DEV)
            hide[:, L:] = ~see.repeat_interleave(G, 0).to(DEV)
            kt = k.transpose(1, 2).contiguous()
            x = torch.matmul(q, kt).masked_fill_(hide, -float("inf"))
            s = torch.matmul(q.abs(), kt.abs()).masked_fill_(hide, 0).amax(2)
            m = x.amax(2, keepdim=True)
            e = (x - m).exp_()
            den = e.sum(2, keepdim=True)
            wo, size, wl = torch.matmul(e, v) / den, torch.matmul(e, v.abs()) / den, (m + den.log())[..., 0]
            r = ((d + 4) * E + 8 * E) * s + 2.0 ** -21
            rest = 2.0 ** -20 + (L + N + 64) * E
            bo = (u + 2 * r + rest)[..., None] * size + u * wo.abs()
            bl = r + rest + 4 * E * wl.abs()
            got_o = o[i, :c].double().view(c, hkv, G, d).transpose(0, 1).reshape(hkv, c * G, d)
            got_l = lse.double().view(hkv, G, n, N)[:, :, i, :c].transpose(1, 2).reshape(hkv, c * G)
            assert ((got_o - wo).abs() <= bo).all(), (i, float(((got_o - wo).abs() / bo).max()))
            assert ((got_l - wl).abs() <= bl).all(), (i, float(((got_l - wl).abs() / bl).max()))
        up = lambda x: (x + 255) // 256 * 256
        at = up(64 * (n + n // self.group)) + up(4 * n * N)
        head = ws[at:at + 32].view(torch.int64).tolist()
        return {"solo": head[:2], "team": head[2:]}


def spread(n, most, least=1, seed=0):
    return [int(x) for x in np.random.default_rng(seed).integers(least, most + 1, n)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,nodes", [(64, 1), (64, 5), (128, 1), (128, 3)])
def test_rings_of_waves(dtype, d, nodes):
    """Many blocks of 32 keys through a wave's ring of two."""
    a = Walk(dtype, 32, 8, d, 64, spread(8, 20000, 17000, d), nodes=nodes, seed=d + nodes)
    assert a.check()["solo"][1] >= 16  # of which 4 are an item's start


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_more_pages_than_a_wave_holds_numbers_of(dtype, d):
    """Runs of more than 64 pages of 16 tokens."""
    a = Walk(dtype, 8, 8, d, 16, spread(8, 44000, 42000, d), seed=d)
    assert a.check()["solo"][1] * 32 > 64 * 16 + 8 * 32


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,nodes", [(64, 1), (64, 4), (128, 2)])
def test_several_items_a_run(dtype, d, nodes):
    """Items of one to four blocks, several to a wave, some without nodes in use."""
    rng = np.random.default_rng(nodes)
    n = 1100
    a = Walk(dtype, 8, 4, d, 16, spread(n, 100, 0, d), nodes=nodes, count=rng.integers(0, nodes + 1, n).tolist() if nodes > 1 else None,
             seed=nodes)
    assert a.check()["solo"][1] >= 9  # an item counts as five to eight


TEAMS = [(32, 8, 64, 12, 1), (32, 8, 128, 12, 1), (32, 8, 64, 40, 1), (32, 8, 128, 40, 1)]  # one tile of rows, two


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d,nodes,group", TEAMS)
def test_rings_of_teams(dtype, hq, hkv, d, nodes, group):
    a = Walk(dtype, hq, hkv, d, 32, spread(4, 24000, 20000, d), nodes=nodes, count=[nodes, nodes - 3, nodes, 34 if nodes > 34 else nodes],
             seed=d + nodes)
    assert a.check()["team"][1] >= 12


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,nodes", [(64, 4), (128, 4), (64, 9), (128, 9)])
def test_groups_of_teams_and_waves(dtype, d, nodes):
    """Shared keys by teams (of one tile of rows, of three), own ones by waves (by teams too), both in long runs."""
    group, G = 8, 4
    lens = [30000 + x for x in spread(2 * group, 3500, 100, d)]
    a = Walk(dtype, 8 * G, 8, d, 64, lens, nodes=nodes, group=group, shared=[460, 468], seed=d + nodes,
             count=[nodes - (i % 3 == 1) for i in range(2 * group)])
    run = a.check()
    assert run["team"][1] >= 8 and (nodes * G > 32 or run["solo"][1] >= 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_of_groups(dtype, d):
    """Shared and own keys by waves, items of very different lengths in one run."""
    group = 8
    lens = [4096 + x for x in spread(6 * group, 500, 0, d)]
    a = Walk(dtype, 32, 8, d, 64, lens, group=group, shared=[64, 60, 64, 1, 64, 0], seed=d)
    assert a.check()["solo"][1] >= 6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nodes", [1, 3, 12])
@pytest.mark.parametrize("rises", [True, False])
def test_maxima_that_rise(dtype, d, nodes, rises):
    """Scores that rise by some 10 in powers of 2 every seven blocks of 32 keys, so that a run rescales what it has; and that
    fall so."""
    a = Walk(dtype, 32, 8, d, 32, spread(4, 27000, 25000, d), nodes=nodes, seed=d + nodes)
    a.q[..., 0] = 4.0
    for i, L in enumerate(a.lens):
        t = torch.arange(a.pages(i).numel() * 32, device=DEV)
        step = (t // 224 if rises else (L + nodes - t).clamp_min(0) // 224).double() * 7.0 / (4.0 * d ** -0.5)
        rows = step.view(-1, 1, 32).expand(-1, 8, -1)
        k = a.k[a.pages(i)]
        k[..., 0] = torch.where(torch.isnan(k[..., 1]), k[..., 1], rows.to(k.dtype))
        a.k[a.pages(i)] = k
    run = a.check()
    assert run["team" if nodes * 4 > 32 else "solo"][1] >= 12
