"""Rows that attend one key: the softmax of one logit is one, so that logit has no gradient.  dQ of such a row is zero and the
row adds nothing to dK, not even a rounding, by whichever kernel the call runs: few tiles, tiles, or a key that is done once
more because a neighbour's values are not finite."""
import pytest
import torch

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}
# few tiles (one launch; two launches), tiles, tiles with shared heads
HEADS = [(2, 2), (40, 40), (140, 140), (256, 32)]


def _step(h, hkv, q, N, d, W, dt, first, spoil=None):
    g = torch.Generator().manual_seed(h + d)
    t = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
    Q, K, V, dO = t(1, h, q, d), t(1, hkv, N, d), t(1, hkv, N, d), t(1, h, q, d)
    if spoil:
        spoil(Q, K, V, dO)
    sh = moba.WindowShape(1, h, q, N, d, window=W, dtype=CODE[dt], kv_heads=hkv)
    O, lse = moba.window_forward(sh, Q, K, V, first_key=first)
    return moba.window_backward(sh, Q, K, V, O, lse, dO, first_key=first)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv", HEADS)
@pytest.mark.parametrize("q,N", [(200, 200), (170, 201)])
def test_sequences_of_one(q, N, h, hkv, dt, d):
    first = torch.arange(N - q, N, dtype=torch.int32).view(1, q).cuda()
    dQ, dK, dV = _step(h, hkv, q, N, d, 40, dt, first)
    assert not dQ.any() and not dK.any()
    assert dV[:, :, N - q:].any(-1).all() and not dV[:, :, :N - q].any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv", HEADS)
def test_sequences_of_one_beside_one_that_is_not_finite(h, hkv, dt, d):
    """Every other row of the tile meets the bad one with a weight of zero, and is done once more."""
    N, at = 200, 77
    first = torch.arange(N, dtype=torch.int32).view(1, N).cuda()

    def spoil(Q, K, V, dO):
        dO[:, :, at] = float("inf")
        Q[:, :, at, 3] = float("nan")

    dQ, dK, dV = _step(h, hkv, N, N, d, 40, dt, first, spoil)
    others = torch.arange(N) != at
    assert not dQ[:, :, others].any() and not dK[:, :, others].any()
    assert dV[:, :, others].any(-1).all()
    # its own values have no finite result
    assert not torch.isfinite(dQ[:, :, at]).any() and not torch.isfinite(dK[:, :, at]).any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv", HEADS)
def test_windows_of_one(h, hkv, dt, d):
    dQ, dK, dV = _step(h, hkv, 131, 131, d, 1, dt, None)
    assert not dQ.any() and not dK.any() and dV.any(-1).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv", HEADS)
def test_sequences_of_one_among_longer_ones(h, hkv, dt, d):
    lens = [1, 1, 30, 1, 65, 1, 1, 40, 1]
    starts = torch.tensor([sum(lens[:i]) for i in range(len(lens))])
    N = sum(lens)
    first = torch.repeat_interleave(starts, torch.tensor(lens)).to(torch.int32).view(1, N).cuda()
    dQ, dK, _ = _step(h, hkv, N, N, d, 70, dt, first)
    ones = [int(s) for s, n in zip(starts, lens) if n == 1]
    assert not dQ[:, :, ones].any() and not dK[:, :, ones].any()
    assert not dQ[:, :, [int(s) for s in starts]].any()
    # (a last key is attended by its own row alone, which attends others: not zero)
    assert dK[:, :, [int(s) + n - 1 for s, n in zip(starts, lens) if n > 1]].any(-1).all()
