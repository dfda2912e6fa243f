"""GPU test of appended rows at positions past 2^20, up to the last that a sequence can have."""
import numpy as np
import pytest
import torch

from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [2**20, 2**20 + 1, 3 * 2**20 + 5, 2**27 + 3, 256 * 8388601 - 4])
def test_positions_past_2_20(d, length):
    """A sequence whose cached pages are not looked at: its new tokens' page alone has a place in the pool.  Angles are 64-bit
    products, reduced with one rounding of pi / 2: off by 2^-53 of the angle twice, and as much again for each turn."""
    ps, hkv, hq, N = 256, 2, 4, 9
    cols = length // ps + 2
    c = pp.Cache(torch.zeros(1, cols, dtype=torch.int32, device=DEV), ints([length]), ints([cols]), ints(np.ones(3)), ps)
    c.page_table[0, length // ps], c.page_table[0, length // ps + 1] = 1, 2
    k, v, q = (wl.randn((1, N, h, d), 5 + h, torch.float32, "cpu") for h in (hkv, hkv + 1, hq))
    v = v[:, :, :hkv].contiguous()
    kp, vp = (torch.zeros(3, hkv, ps, d, device=DEV) for _ in range(2))
    q_rot = pp.pp_cache_append(c, ints([0]), k.to(DEV), v.to(DEV), kp, vp, q=q.to(DEV), rope_base=1e4).cpu().double().numpy()
    for j in range(N):
        t = length + j
        page, row = 1 + t // ps - length // ps, t % ps
        angle = t * 2.0 ** -51 * 2  # of the fastest pair, t radians
        for got, x in ((kp[page, :, row], k[0, j]), (q_rot[0, j], q[0, j])):
            x = x.double().numpy()
            want = smp.rotate(x, t, 1e4)
            got = got.double().cpu().numpy() if torch.is_tensor(got) else got
            size = np.abs(x[:, :d // 2]) + np.abs(x[:, d // 2:])
            size = np.concatenate([size, size], axis=1)
            # cos and sin to 2^-23 (an angle rounded to fp32, a series in it), products and their sum
            assert (np.abs(got - want) <= size * (angle + 6 * 2.0 ** -24) + 2.0 ** -24 * np.abs(want)).all(), (j, np.abs(got - want).max())
        np.testing.assert_array_equal(vp[page, :, row].cpu().numpy(), v[0, j].numpy())


def test_accept_goes_by_a_slots_first_entry():
    """Also where that one keeps nothing."""
    c = pp.Cache(ints(np.zeros((3, 2))), ints([4, 4, 4]), ints([1, 1, 1]), ints(np.zeros(4)), 16)
    slots, count = [0, 0, 1, 9, -1], [0, 3, 2, 0, 5]
    b = smp.Book(np.zeros((3, 2)), [4, 4, 4], [1, 1, 1], np.zeros(4), 16)
    assert pp.pp_cache_accept(c, ints(slots), ints(count)).tolist() == b.accept(slots, count) == [0, 1]
    assert c.seq_len.tolist() == b.len.tolist() == [4, 6, 4]
