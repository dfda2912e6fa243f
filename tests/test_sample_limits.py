"""CPU tests of the sampling operators' largest sizes: what no launch can take is refused ahead of the first; and of which entry of
a call counts."""
import ctypes

import numpy as np
import pytest

from oracle import sampling as smp
from paper_2602_24082_amd import binding as pp

OK = ctypes.c_void_p(4096)
DESC = pp._CacheDesc(4, 8, 32, 16, OK, OK, OK, OK)


def _tree(n, nodes, hq, d):
    """pp_tree_attn_fwd's answer: 3 too large, 4 the workspace is too small (all else is fine)."""
    return pp.lib().pp_tree_attn_fwd(ctypes.byref(DESC), n, OK, 1, None, nodes, None, None, pp.PP_BF16, hq, 1, d, 0.0, OK, OK, OK, OK,
                                     OK, 0, OK, 64, None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nodes,hq,status", [
    (2040, 39, 1687, 4),  # 2^27 - 8 rows: the join's 2^24 - 1 workgroups of 256 threads
    (1801, 31, 2404, 3),  # 2^27 - 4: one workgroup more, 2^32 threads
    (2048, 16, 4096, 3),  # 2^27
])
def test_rows_that_the_join_cannot_launch(d, n, nodes, hq, status):
    rows = n * nodes * hq
    assert (rows + 7) // 8 * 256 < 2**32 or status == 3
    assert _tree(n, nodes, hq, d) == status
    size = ctypes.c_size_t(0)
    assert pp.lib().pp_tree_workspace_size(ctypes.byref(DESC), n, 1, nodes, pp.PP_BF16, hq, 1, d, ctypes.byref(size)) == (3 if status == 3 else 0)


def test_oracle_accepts_by_a_slots_first_entry():
    """A slot named twice counts by its first entry, also where that one keeps nothing."""
    b = smp.Book(np.zeros((3, 2)), [4, 4, 4], [1, 1, 1], np.zeros(4), 16)
    assert b.accept([0, 0, 1, 9, -1], [0, 3, 2, 0, 5]) == [0, 1]
    assert b.len.tolist() == [4, 6, 4]
