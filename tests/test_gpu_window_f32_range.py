"""fp32 numbers of all sizes through products of three bf16 parts.  Where a row attends one key its weight is one and O is the
key's value: to the bit, as far down as the three parts hold 24 bits, and below 2^-108 to within what the last part
loses, which is less than 2^-126 (a part below that may be lost)."""
import pytest
import torch

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu


def _numbers(n, d, low, high):
    """Every binade from 2^low to 2^high, either sign, 24 random bits."""
    g = torch.Generator().manual_seed(n + d)
    e = torch.randint(low, high, (n * d,), generator=g)
    m = 1.0 + torch.randint(0, 1 << 23, (n * d,), generator=g).double() * 2.0 ** -23
    s = 1.0 - 2.0 * torch.randint(0, 2, (n * d,), generator=g).double()
    x = s * m * torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double())
    return x.float()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h", [1, 40, 140])                   # few tiles, one launch and two; tiles
def test_values_of_all_sizes(h, d):
    N = 131
    sh = moba.WindowShape(1, h, N, N, d, window=1, dtype=binding.F32)
    Q, K = torch.zeros((2, 1, h, N, d), device="cuda")
    V = _numbers(h * N, d, -108, 128).view(1, h, N, d).cuda()
    O, lse = moba.window_forward(sh, Q, K, V)
    assert torch.equal(O, V) and not lse.any()
    dQ, dK, dV = moba.window_backward(sh, Q, K, torch.zeros_like(V), torch.zeros_like(V), lse, V)
    assert torch.equal(dV, V) and not dQ.any() and not dK.any()
    small = _numbers(h * N, d, -126, -108).view(1, h, N, d).cuda()
    O, _ = moba.window_forward(sh, Q, K, small)
    assert ((O.double() - small.double()).abs() <= 2.0 ** -126).all()
