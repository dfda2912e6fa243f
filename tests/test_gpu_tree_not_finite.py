"""GPU tests of the attention over the paged cache where drafted nodes are not finite: they reach the nodes that see them, in the
elements where they do by the definition, and leave the others as exact as ever (test_gpu_tree.py's bounds)."""
import numpy as np
import pytest
import torch

from oracle import sampling as smp
from test_gpu_tree import DEV, E, U, Case, ints

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def put(a, pool, i, node, x, head=0, dims=slice(None)):
    """Sets elements of a node's row."""
    t = int(a.cache.seq_len[a.slots[i]]) + node
    ps = a.cache.page_size
    pool[int(a.cache.page_table[a.slots[i], t // ps]), head, t % ps, dims] = x


def check(a, chains=False):
    o, lse = (x.double().cpu().numpy() for x in a.run(chains))
    n64 = lambda t: t.double().numpy()[None]
    b = smp.Book(a.cache.page_table.cpu().numpy(), a.cache.seq_len.cpu().numpy(), a.cache.held.cpu().numpy(), [], a.cache.page_size,
                 n64(a.k), n64(a.v))
    u, d = U[a.dtype], a.q.shape[3]
    with np.errstate(invalid="ignore"):
        wo, wl, size, s = smp.tree_attn(b, 0, a.slots, a.q.double().numpy(), None if chains else a.parents, a.count)
    N = int(max(b.len)) + a.nodes
    r = ((d + 4) * E + 8 * E) * s + 2.0 ** -21
    for name, got, want in (("o", o, wo), ("lse", lse, wl)):
        np.testing.assert_array_equal(np.isfinite(got), np.isfinite(want), err_msg=name)
    ok = np.isfinite(wo)
    bo = (u + 2 * r + 2.0 ** -20 + (N + 64) * E)[..., None] * size + u * np.abs(wo)
    assert (np.abs(o[ok] - wo[ok]) <= bo[ok]).all()
    ok = np.isfinite(wl)
    bl = (r + 2.0 ** -20 + (N + 64) * E).transpose(2, 0, 1).reshape(wl.shape) + 4 * E * np.abs(wl)
    assert (np.abs(lse[ok] - wl[ok]) <= bl[ok]).all()
    return o


# solo waves; teams of one tile of rows and of two
SHAPES = [(4, 2, 64, 7), (14, 2, 64, 4), (8, 2, 128, 7), (8, 1, 128, 9), (16, 1, 64, 7), (8, 1, 64, 20), (4, 1, 128, 40)]
LENS = [0, 5, 27, 31, 32, 57, 500]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,nodes", SHAPES)
@pytest.mark.parametrize("x", [NAN, INF, -INF])
def test_values_of_a_branch(dtype, hq, hkv, d, nodes, x):
    """A leaf that is another branch's sibling; the last node in use, whose row stands in for what lies behind it; one element
    only; the first node of all."""
    a = Case(dtype, hq, hkv, d, 16, LENS, nodes=nodes, count=[nodes] * 5 + [nodes - 1] * 2, seed=nodes + d)
    a.parents = [[-1, 0, 0] + [2 if j % 2 else j - 2 for j in range(3, nodes)]] * len(LENS)
    put(a, a.v, 0, 1, x)
    put(a, a.v, 1, nodes - 1, x)
    put(a, a.v, 2, 1, x, head=hkv - 1, dims=d - 1)
    put(a, a.v, 3, 0, x, dims=3)
    put(a, a.v, 4, nodes - 1, x, head=hkv - 1, dims=slice(5, 40, 7))
    put(a, a.v, 5, nodes - 2, x)
    put(a, a.v, 6, 1, x)
    put(a, a.v, 6, 2, -x, dims=2)
    o = check(a)
    assert np.isfinite(o[0, 0]).all() and not np.isfinite(o[0, 1]).all() and not np.isfinite(o[3, -1]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,nodes", SHAPES)
def test_keys_and_queries_of_a_branch(dtype, hq, hkv, d, nodes):
    a = Case(dtype, hq, hkv, d, 16, LENS, nodes=nodes, seed=nodes + d)
    a.parents = [[-1, 0, 0] + [2 if j % 2 else j - 2 for j in range(3, nodes)]] * len(LENS)
    for i in range(len(LENS)):
        put(a, a.k, i, [1, nodes - 1, 1, 0, 2, nodes - 1, 1][i], NAN, dims=i)
    a.q[0, 2, 0, 3] = NAN
    a.q[5, 0, -1, 0] = INF
    check(a)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_chain_and_shared_pages(dtype):
    """A chain's later nodes are not seen by its earlier ones; a group's shared pages end inside a block of keys."""
    for hq, hkv, d, nodes in ((4, 2, 64, 6), (8, 1, 128, 12)):
        a = Case(dtype, hq, hkv, d, 16, [50, 55, 48, 16, 20, 31], group=3, shared=[3, 1], nodes=nodes, seed=d)
        for i in range(6):
            put(a, a.v, i, [3, nodes - 1, 1, 0, 4, 2][i], NAN, head=hkv - 1, dims=slice(0, d, 9))
        o = check(a, chains=True)
        assert np.isfinite(o[0, :3]).all() and not np.isfinite(o[0, 3]).all() and not np.isfinite(o[0, -1]).all()
        put(a, a.v, 3, -9, INF, dims=1)  # a key that all see
        o = check(a, chains=True)
        assert not np.isfinite(o[3, :, 0, 1]).any()


def test_values_above_what_bf16_holds():
    """fp32 values that round to infinity as bf16 stay with those that see them."""
    a = Case(torch.float32, 4, 2, 64, 16, [5, 40], nodes=4, seed=3)
    a.parents = [[-1, 0, 0, 0]] * 2
    for i in range(2):
        put(a, a.v, i, 2, 3.4e38, dims=7)
    o, _ = a.run()
    o = o.cpu()
    bad = ~torch.isfinite(o)
    assert bad[:, 2, :2, 7].all() and bad.sum() == 2 * 2
