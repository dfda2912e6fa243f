"""GPU tests of the log-prob gradient with entropies on rows in which some values lie far
above what a wave looks at first (its threads' first vectors, the base of its sums), and
on rows whose first vectors are masked with finite numbers.  Bounds: test_gpu_policy.py's,
which allow for an exponent's rounding over the whole distance."""
import pytest
import torch

from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl
from test_gpu_policy import DEV, _check_tok, _pack

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
# threads x vectors that hold a row: 512 x 8, 1024 x 8, 1024 x 19, off the boundaries 1024 x 18, streamed past 1024 x 16
SHAPES = [(16000, F32), (32000, BF), (30001, F32), (65536, BF), (152064, BF), (147450, BF), (163840, BF), (155661, BF)]


def _first(V, dtype):
    """Elements that the threads' first vectors hold, at most."""
    n = 16 // (torch.finfo(dtype).bits // 8)
    return (512 if V // n <= 4096 else 1024) * n + n


def _case(V, dtype, seed):
    """Rows of values in (-3, 0): some first vector of every wave comes within 0.1 of 0."""
    pack = _pack()
    T = pack.total_tokens
    x = (-3.0 * torch.rand((T, V), generator=torch.Generator().manual_seed(seed))).to(dtype)
    return (pack, x, wl.randint((T,), V, seed + 1, "cpu"), wl.randn((T,), seed + 2, F32, "cpu"), wl.randn((T,), seed + 3, F32, "cpu"))


def _both(pack, x, y, g, h):
    _check_tok(pack, x, y, g, h)
    _check_tok(pack, x, y, g, torch.zeros_like(h))  # the weights of no entropy: the log-probs' gradient stands


@pytest.mark.parametrize("gap", [20.0, 60.0, 80.0, 83.5, 84.5, 86.0, 88.0, 88.5, 89.5, 92.0])
@pytest.mark.parametrize("V,dtype", SHAPES)
def test_peak_past_the_first_vectors(V, dtype, gap):
    """e^gap times the gap's exponent overflows ahead of e^gap itself, between 84 and 88.7."""
    pack, x, y, g, h = _case(V, dtype, 700)
    x[:, _first(V, dtype) + V // 7] = gap
    y[4] = _first(V, dtype) + V // 7
    _both(pack, x, y, g, h)


@pytest.mark.parametrize("gap,high", [(86.0, 290.0), (86.0, 86.5), (87.0, 88.5), (87.5, 88.5), (60.0, 89.0), (100.0, 101.0)])
@pytest.mark.parametrize("V,dtype", SHAPES)
def test_peak_beside_a_wave_with_a_higher_base(V, dtype, gap, high):
    """Another wave's first vectors hold `high`: with 290 the peak has no weight, a little above the gap
    both have, though the peak's wave counts from a base so far below that 2^-127 of it is 0 in fp32."""
    pack, x, y, g, h = _case(V, dtype, 720)
    at = _first(V, dtype) + 70 * 16 // (torch.finfo(dtype).bits // 8)  # not of the first wave
    x[:, 9] = high
    x[:, at] = gap
    y[3], y[4] = 9, at
    _both(pack, x, y, g, h)


@pytest.mark.parametrize("value", [-1e4, -65504.0, -1e9, -1e29, float("-inf")])
@pytest.mark.parametrize("V,dtype", SHAPES)
def test_masked_first_vectors(V, dtype, value):
    pack, x, y, g, h = _case(V, dtype, 740)
    n = _first(V, dtype)
    y = n + y % (V - n)
    x[:, :n] = value
    _both(pack, x, y, g, h)
    # of some waves only
    x[:, :n // 3] = -1.0
    _both(pack, x, y, g, h)


@pytest.mark.parametrize("V,dtype", [(16000, F32), (152064, BF), (163840, BF)])
def test_runs_agree_bit_for_bit(V, dtype):
    pack, x, y, g, h = _case(V, dtype, 760)
    x[:, _first(V, dtype) + V // 7] = 86.0
    a, b = (pp.pp_tok_logprob_bwd(pack, *(t.to(DEV) for t in (x, y, g, h))) for _ in range(2))
    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
