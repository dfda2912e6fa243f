"""GPU tests of the paged cache against the oracle's, page by page: tables, counts and moved rows bit for bit, rotated rows
within their rounding; slots named twice, entries that are no slot, unsound lengths, pages that are none, a pool that runs out."""
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


def pools(layers, pages, hkv, ps, d, dtype, seed):
    return [wl.randn((layers, pages, hkv, ps, d), seed + i, dtype, "cpu").to(DEV) for i in range(2)]


def book_of(cache, k, v):
    """The oracle's copy of what is on the GPU (values in 64 bits: bf16 and fp32 numbers as they are)."""
    n = lambda t: t.cpu().numpy()
    return smp.Book(n(cache.page_table), n(cache.seq_len), n(cache.held), n(cache.refs), cache.page_size,
                    k.double().cpu().numpy(), v.double().cpu().numpy())


def same(cache, k, v, book):
    torch.cuda.synchronize()
    for name, t, want in (("table", cache.page_table, book.table), ("len", cache.seq_len, book.len), ("held", cache.held, book.held),
                          ("refs", cache.refs, book.refs), ("k", k.double(), book.pools[0]), ("v", v.double(), book.pools[1])):
        np.testing.assert_array_equal(t.cpu().numpy(), want, err_msg=name)


def junk_ws(cache, n):
    return torch.full((pp.pp_cache_workspace_size(cache, n),), 0xff, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("dtype,ps,hkv,d,layers", [(torch.bfloat16, 16, 2, 64, 3), (torch.float32, 32, 3, 128, 1),
                                                   (torch.bfloat16, 256, 1, 128, 2), (torch.float32, 64, 8, 64, 2)])
def test_a_life_of_a_cache(dtype, ps, hkv, d, layers):
    """Every call in turn on one cache, with entries that are refused among them."""
    rng = np.random.default_rng(ps + hkv)
    slots, cols, pages = 23, 7, 60
    c = pp.make_cache(slots, cols, pages, ps, DEV)
    k, v = pools(layers, pages, hkv, ps, d, dtype, 5)
    b = book_of(c, k, v)
    st = lambda s: s.cpu().tolist()
    lens = [3 * ps + 5, ps, 1, 2 * ps - 1]
    args = [0, 1, 2, 3, 1, -1, slots, 5], lens + [4, 9, 9, -1]
    assert st(pp.pp_cache_reserve(c, ints(args[0]), ints(args[1]), ws=junk_ws(c, 8))) == b.reserve(*args) == [0, 3]
    assert st(pp.pp_cache_accept(c, ints([0, 1, 2, 3]), ints(lens))) == b.accept([0, 1, 2, 3], lens) == [0, 0]
    same(c, k, v, b)
    src, dst = [0, 0, 0, 1, 2, 3, 3, -1, 0, 0, 7, 3], [10, 11, 12, 13, 14, 15, 16, -1, 11, 1, 17, slots + 2]
    assert st(pp.pp_cache_fork(c, ints(src), ints(dst), k, v, ws=junk_ws(c, 12))) == b.fork(src, dst) == [0, 3]
    same(c, k, v, b)
    assert pp.pp_cache_shared(c, ints([10, 11, 12, 0, 13, 14, 15, 16, -1, 5, -1, 4]), 4).cpu().tolist() == \
        b.shared([10, 11, 12, 0, 13, 14, 15, 16, -1, 5, -1, 4], 4)
    pp.pp_cache_free(c, ints([0, 0, 3, -5, 2, slots]))
    b.free([0, 0, 3, -5, 2, slots])
    same(c, k, v, b)
    add = rng.integers(1, ps, size=6).tolist()
    grow = [10, 11, 12, 13, 15, 16]
    assert st(pp.pp_cache_reserve(c, ints(grow), ints(add))) == b.reserve(grow, add)
    pp.pp_cache_free(c, ints([11, 13]))
    b.free([11, 13])
    assert pp.pp_cache_compact(c, k, v, ws=junk_ws(c, 0)).cpu().tolist() == [b.compact()]
    same(c, k, v, b)
    # the pool runs out: nothing changes
    many = list(range(17, 23)) + [0, 2, 3, 11]
    want = b.reserve(many, [ps * cols] * 10)
    assert st(pp.pp_cache_reserve(c, ints(many), ints([ps * cols] * 10))) == want and want[0] > 0
    assert st(pp.pp_cache_reserve(c, ints([17]), ints([ps * cols + 1]))) == b.reserve([17], [ps * cols + 1]) == [0, 1]
    same(c, k, v, b)
    pp.pp_cache_free(c, ints(list(range(slots))))
    b.free(list(range(slots)))
    assert pp.pp_cache_compact(c, k, v).cpu().tolist() == [b.compact()] == [0]
    same(c, k, v, b)


def test_fork_runs_out():
    c = pp.make_cache(8, 4, 5, 16, DEV)
    k, v = pools(1, 5, 1, 16, 64, torch.bfloat16, 1)
    pp.pp_cache_reserve(c, ints([0]), ints([40]))
    pp.pp_cache_accept(c, ints([0]), ints([40]))
    b = book_of(c, k, v)
    args = [0, 0, 0, 0], [1, 2, 3, 4]
    assert pp.pp_cache_fork(c, ints(args[0]), ints(args[1]), k, v).cpu().tolist() == b.fork(*args) == [2, 0]
    same(c, k, v, b)


def test_fork_of_what_the_same_call_fills():
    """The state ahead of the call counts: a source that another entry fills is empty."""
    for order in (1, -1):
        c = pp.make_cache(400, 4, 900, 16, DEV)
        k, v = pools(1, 900, 1, 16, 64, torch.bfloat16, 2)
        pp.pp_cache_reserve(c, ints([0]), ints([40]))
        pp.pp_cache_accept(c, ints([0]), ints([40]))
        b = book_of(c, k, v)
        src, dst = [0] + list(range(1, 300)), list(range(1, 301))
        args = src[::order], dst[::order]
        assert pp.pp_cache_fork(c, ints(args[0]), ints(args[1]), k, v).cpu().tolist() == b.fork(*args) == [0, 0]
        same(c, k, v, b)


def test_many_slots():
    """More slots than a workgroup marks in LDS."""
    n = 9000
    c = pp.make_cache(n, 2, 400, 16, DEV)
    k, v = pools(1, 400, 1, 16, 64, torch.bfloat16, 4)
    b = book_of(c, k, v)
    slots = [n - 1 - i for i in range(0, 1200, 7)] + [n - 1, 5, n]
    add = [1 + i % 20 for i in range(len(slots))]
    assert pp.pp_cache_reserve(c, ints(slots), ints(add), ws=junk_ws(c, len(slots))).cpu().tolist() == b.reserve(slots, add) == [0, 2]
    assert pp.pp_cache_accept(c, ints(slots), ints(add)).cpu().tolist() == b.accept(slots, add) == [0, 2]
    src = slots[:20]
    assert pp.pp_cache_fork(c, ints(src), ints([i % 18 for i in range(20)]), k, v).cpu().tolist() == b.fork(src, [i % 18 for i in range(20)])
    same(c, k, v, b)


def test_large_pool():
    """More pages than one round of the search looks at, free ones far apart; many entries."""
    pages, n = 30011, 1500
    rng = np.random.default_rng(3)
    refs = (rng.random(pages) < 0.9).astype(np.int32)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    c = pp.Cache(z(2 * n, 3), z(2 * n), z(2 * n), ints(refs), 16)
    k, v = (torch.zeros(1, pages, 1, 16, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[0, :, 0, :, 0] = torch.arange(pages, device=DEV)[:, None] % 251
    b = book_of(c, k, v)
    add = rng.integers(0, 33, size=n).tolist()
    assert pp.pp_cache_reserve(c, ints(range(n)), ints(add)).cpu().tolist() == b.reserve(list(range(n)), add) == [0, 0]
    assert pp.pp_cache_accept(c, ints(range(n)), ints(add)).cpu().tolist() == b.accept(list(range(n)), add)
    src = list(range(400))
    assert pp.pp_cache_fork(c, ints(src), ints([n + s for s in src]), k, v).cpu().tolist() == b.fork(src, [n + s for s in src])
    same(c, k, v, b)
    pp.pp_cache_free(c, ints(range(0, n, 2)))
    b.free(range(0, n, 2))
    # pages that nobody lists go too: only those of the cache are followed by tables
    assert pp.pp_cache_compact(c, k, v).cpu().tolist() == [b.compact()]
    same(c, k, v, b)


def _append_case(dtype, ps, hkv, d, layers=1, seed=0):
    c = pp.make_cache(9, 8, 40, ps, DEV)
    k, v = pools(layers, 40, hkv, ps, d, dtype, seed)
    pp.pp_cache_reserve(c, ints([0, 2, 5, 7]), ints([ps + 3, 1, 2 * ps, 5]))
    pp.pp_cache_accept(c, ints([0, 2, 5, 7]), ints([ps + 3, 1, 2 * ps, 5]))
    return c, k, v


def _turned(x, pos, base, dtype):
    """(the rotated rows, their error's bound): one rounding to the type, fp32 products, sines good to 1e-7."""
    y = smp.rotate(x, pos, base)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    return y, half * np.abs(y) + 4e-6 * np.abs(x).max()


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ps,hq,hkv,d", [(16, 4, 2, 64), (32, 6, 3, 128), (64, 32, 8, 128), (16, 71, 1, 64)])
def test_append_tree(dtype, base, ps, hq, hkv, d):
    c, kp, vp = _append_case(dtype, ps, hkv, d)
    slots, N = [5, 0, -1, 7, 2, 20], 6
    count, parents = [6, 3, 6, 0, 4, 2], [[-1, 0, 0, 1, 1, 3], [-1, -1, 0, 0, 0, 0], [-1] * 6, [-1] * 6, [-1, 0, 1, 2, 9, 9], [-1] * 6]
    pp.pp_cache_reserve(c, ints([5, 0, 2]), ints([6, 3, 4]))
    b = book_of(c, kp, vp)
    k, v, q = (wl.randn((6, N, h, d), 30 + h, dtype, "cpu") for h in (hkv, hkv, hq))
    qr = torch.full(q.shape, float("nan"), dtype=dtype, device=DEV)
    pp.pp_cache_append(c, ints(slots), k.to(DEV), v.to(DEV), kp[0], vp[0], count=ints(count), parents=ints(parents), q=q.to(DEV),
                       rope_base=base, q_rot=qr)
    torch.cuda.synchronize()
    bound = np.zeros(b.pools[0].shape)
    want_q, bq = np.zeros(q.shape), np.zeros(q.shape)
    for i, s in enumerate(slots):
        for j, dep in enumerate(smp.depths(parents[i])[:count[i] if s >= 0 else 0]):
            pos = (int(b.len[s]) if s < 9 else 0) + dep
            x, y = k[i, j].double().numpy(), q[i, j].double().numpy()
            (kr, bk), (want_q[i, j], bq[i, j]) = ((_turned(x, pos, base, dtype), _turned(y, pos, base, dtype)) if base
                                                  else ((x, 0 * x), (y, 0 * y)))
            if s < 9:
                b.append(0, s, j, kr, v[i, j].double().numpy())
                p, r = b.place(s, int(b.len[s]) + j)
                bound[0, p, :, r] = bk
    assert (np.abs(kp.double().cpu().numpy() - b.pools[0]) <= bound).all()
    np.testing.assert_array_equal(vp.double().cpu().numpy(), b.pools[1])
    assert (np.abs(qr.double().cpu().numpy() - want_q) <= bq).all()


def test_append_prompts_of_a_packed_batch():
    """start and count from a packed batch: prompts of different lengths, one without pages for all of it; far positions."""
    pack = wl.make_pack([33, 7, 64], [[3, 2], [], [5]], pad=[2, 0, 1])
    T, hkv, hq, d, ps = pack.total_tokens, 2, 4, 64, 16
    c = pp.make_cache(5, 6, 20, ps, DEV)
    kp, vp = pools(1, 20, hkv, ps, d, torch.float32, 3)
    pp.pp_cache_reserve(c, ints([4, 1, 0]), ints([33, 7, 40]))  # 48 of 64
    b = book_of(c, kp, vp)
    k, v, q = (wl.randn((T, h, d), 40 + i, torch.float32, "cpu") for i, h in enumerate((hkv, hkv, hq)))
    qd = q.to(DEV)
    pp.pp_cache_append(c, ints([4, 1, 0]), k.to(DEV), v.to(DEV), kp[0], vp[0], count=ints(pack.prompt_len),
                       start=ints(pack.row_start[:-1]), max_new=64, q=qd, rope_base=500.0, q_rot=qd)
    want_q, bq = q.double().numpy().copy(), np.zeros(q.shape)  # rows of responses and padding stay
    bound = np.zeros(b.pools[0].shape)
    for i, s in enumerate([4, 1, 0]):
        for j in range(int(pack.prompt_len[i])):
            t = int(pack.row_start[i]) + j
            want_q[t], bq[t] = _turned(q[t].double().numpy(), j, 500.0, torch.float32)
            kr, bk = _turned(k[t].double().numpy(), j, 500.0, torch.float32)
            b.append(0, s, j, kr, v[t].double().numpy())
            if j < b.held[s] * ps:
                p, r = b.place(s, j)
                bound[0, p, :, r] = bk
    assert (np.abs(qd.double().cpu().numpy() - want_q) <= bq).all()
    assert (np.abs(kp.double().cpu().numpy() - b.pools[0]) <= bound).all()
    np.testing.assert_array_equal(vp.double().cpu().numpy(), b.pools[1])
    # rows past the tensors are not read: the last token's start lies behind them
    pp.pp_cache_append(c, ints([4]), k.to(DEV), v.to(DEV), kp[0], vp[0], count=ints([10]), start=ints([T - 2]), max_new=10)
    for j in range(2):
        b.append(0, 4, j, k[T - 2 + j].double().numpy(), v[T - 2 + j].double().numpy())
        p, r = b.place(4, j)
        bound[0, p, :, r] = 0
    assert (np.abs(kp.double().cpu().numpy() - b.pools[0]) <= bound).all()


def test_append_far_positions():
    """Angles of positions past 2^20 (64 bits), in a cache that holds little."""
    c = pp.make_cache(1, 1 << 16, 4, 16, DEV)
    c.held.fill_((1 << 16))
    c.seq_len.fill_((1 << 20) - 5)
    c.page_table.fill_(2)
    kp, vp = pools(1, 4, 1, 16, 128, torch.float32, 8)
    k, v = (wl.randn((1, 5, 1, 128), 50 + i, torch.float32, "cpu") for i in range(2))
    pp.pp_cache_append(c, ints([0]), k.to(DEV), v.to(DEV), kp[0], vp[0], rope_base=1e6)
    for j in range(5):
        want, bound = _turned(k[0, j].double().numpy(), (1 << 20) - 5 + j, 1e6, torch.float32)
        assert (np.abs(kp[0, 2, :, 11 + j].double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ps,hkv,d,N", [(16, 2, 64, 5), (16, 3, 128, 64), (64, 1, 64, 33)])
def test_accept(dtype, ps, hkv, d, N):
    rng = np.random.default_rng(N)
    c, kp, vp = _append_case(dtype, ps, hkv, d, layers=2, seed=9)
    slots = [0, 2, 5, 7, 0, -1, 3, 2]
    pp.pp_cache_reserve(c, ints([0, 2, 5, 7]), ints([N, N, N, N // 2]))
    path = np.full((8, N), -1)
    count = [N // 2, N, 3, N // 2, 1, 1, 1, 1]
    for i, m in enumerate(count):
        path[i, :m] = np.sort(rng.permutation(N)[:m])
    path[2, :3] = [0, 2, 1]         # does not ascend
    path[3, N // 2 - 1] = N - 1     # may leave the reserved pages
    b = book_of(c, kp, vp)
    got = pp.pp_cache_accept(c, ints(slots), ints(count), ints(path), kp, vp, ws=junk_ws(c, 8))
    assert got.cpu().tolist() == b.accept(slots, count, path, N)
    same(c, kp, vp, b)


def test_pages_that_are_none():
    """Table entries outside the pool: rows there are neither written nor moved, references not touched."""
    c, kp, vp = _append_case(torch.bfloat16, 16, 2, 64)
    pp.pp_cache_reserve(c, ints([5]), ints([20]))
    c.page_table[5, 2] = 1 << 20  # of the places 32 ..
    c.page_table[0, 1] = -7
    b = book_of(c, kp, vp)
    k = wl.randn((1, 20, 2, 64), 3, torch.bfloat16, "cpu")
    pp.pp_cache_append(c, ints([5]), k.to(DEV), k.to(DEV), kp[0], vp[0])
    for j in range(20):
        b.append(0, 5, j, k[0, j].double().numpy(), k[0, j].double().numpy())
    assert pp.pp_cache_fork(c, ints([0, 5]), ints([1, 3]), kp, vp).cpu().tolist() == b.fork([0, 5], [1, 3]) == [0, 1]
    path = [[0, 18]]
    assert pp.pp_cache_accept(c, ints([5]), ints([2]), ints(path + [])[:, :2].contiguous(), kp, vp).cpu().tolist() == [0, 1]
    pp.pp_cache_free(c, ints([5, 0]))
    b.free([5, 0])
    same(c, kp, vp, b)


def test_unsound_lengths_are_refused():
    c, kp, vp = _append_case(torch.bfloat16, 16, 2, 64)
    c.seq_len[0] = 1000
    c.held[5] = 99
    c.seq_len[7] = -3
    b = book_of(c, kp, vp)
    assert pp.pp_cache_reserve(c, ints([0, 5, 7, 2]), ints([1, 1, 1, 1])).cpu().tolist() == b.reserve([0, 5, 7, 2], [1] * 4) == [0, 3]
    assert pp.pp_cache_fork(c, ints([0, 5, 7]), ints([1, 3, 4]), kp, vp).cpu().tolist() == b.fork([0, 5, 7], [1, 3, 4]) == [0, 3]
    assert pp.pp_cache_accept(c, ints([0, 5, 7]), ints([1, 1, 1])).cpu().tolist() == b.accept([0, 5, 7], [1] * 3) == [0, 3]
    assert pp.pp_cache_shared(c, ints([0, 5]), 2).cpu().tolist() == [0]
    x = torch.ones(3, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    pp.pp_cache_append(c, ints([0, 5, 7]), x, x, kp[0], vp[0])
    same(c, kp, vp, b)


def test_no_entries():
    """Calls of no sequences: the statuses say so and nothing changes."""
    c, kp, vp = _append_case(torch.bfloat16, 16, 2, 64)
    b, none = book_of(c, kp, vp), ints([])
    assert pp.pp_cache_reserve(c, none, none).tolist() == [0, 0]
    assert pp.pp_cache_fork(c, none, none, kp, vp).tolist() == [0, 0]
    assert pp.pp_cache_accept(c, none, none).tolist() == [0, 0]
    assert pp.pp_cache_accept(c, none, none, ints(np.zeros((0, 4))), kp, vp).tolist() == [0, 0]
    pp.pp_cache_free(c, none)
    x = torch.ones(0, 4, 2, 64, dtype=torch.bfloat16, device=DEV)
    pp.pp_cache_append(c, none, x, x, kp[0], vp[0])
    assert pp.pp_cache_shared(c, none, 3).tolist() == []
    same(c, kp, vp, b)


def test_binding_refuses():
    c, kp, vp = _append_case(torch.bfloat16, 16, 2, 64)
    x = torch.ones(1, 3, 2, 64, dtype=torch.bfloat16, device=DEV)
    one = ints([0])
    for bad in (lambda: pp.pp_cache_append(c, one, x, x, kp, vp[0]), lambda: pp.pp_cache_append(c, one, x[:, ::2], x[:, ::2], kp[0], vp[0]),
                lambda: pp.pp_cache_append(c, one, x.float(), x, kp[0], vp[0]), lambda: pp.pp_cache_append(c, one.long(), x, x, kp[0], vp[0]),
                lambda: pp.pp_cache_append(c, one, x.cpu(), x, kp[0], vp[0]), lambda: pp.pp_cache_append(c, one, x[0], x[0], kp[0], vp[0]),
                lambda: pp.pp_cache_fork(c, one, ints([1, 2]), kp, vp), lambda: pp.pp_cache_reserve(c, one.cpu(), one),
                lambda: pp.pp_cache_accept(c, one, one, ints([[0, 1]])), lambda: pp.pp_cache_shared(c, ints([0, 1, 2]), 2)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    with pytest.raises(pp.PPError):
        pp.make_cache(4, 4, 4, 24, DEV) and pp.pp_cache_free(pp.make_cache(4, 4, 4, 24, DEV), one)
