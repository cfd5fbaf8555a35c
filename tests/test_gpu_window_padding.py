"""Padded batches: what the padding holds -- keys, values, queries and gradients that no pair has, uninitialised memory say --
does not change a bit of any result, nor is it read."""
import pytest
import torch

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}

# batch, heads, kv heads, q_len, kv_len, window: few tiles (one launch, two, shared heads, keys shared by workgroups), tiles, tokens of a cache
CASES = [(3, 2, 2, 230, 230, 0), (3, 2, 1, 230, 230, 50), (3, 20, 20, 230, 230, 0), (3, 40, 40, 230, 230, 60), (3, 56, 28, 230, 230, 0),
         (2, 1, 1, 1300, 1300, 0), (3, 4, 2, 1, 1700, 0), (3, 8, 2, 5, 300, 0), (3, 64, 64, 150, 330, 90)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side", ["left", "right", "both"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_padding_changes_no_bit(case, side, dt, d):
    b, h, hkv, q, N, W = case
    g = torch.Generator().manual_seed(sum(case) + d)
    t = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
    Q, K, V, dO = t(b, h, q, d), t(b, hkv, N, d), t(b, hkv, N, d), t(b, h, q, d)
    pos, keys = torch.arange(N - q, N), torch.arange(N)
    first, real = torch.zeros((b, q), dtype=torch.int32), torch.ones((b, N), dtype=torch.bool)
    for i in range(b):
        begin = [70, 0, 97][i] if side != "right" else 0
        end = N if side == "left" or q < 32 else N - [45, 100, 0][i]
        first[i] = torch.where((pos >= begin) & (pos < end), begin, [1 << 30, 2 ** 31 - 1, N][i])
        real[i] = (keys >= begin) & (keys < end)
    first, pad_k, pad_q = first.cuda(), ~real[:, None].expand(b, hkv, N), ~real[:, None, N - q:].expand(b, h, q)
    sh = moba.WindowShape(b, h, q, N, d, window=W, dtype=CODE[dt], kv_heads=hkv)
    out = []
    for key, value, query, grad in ((0.0, 0.0, 0.0, 0.0), (float("nan"), float("nan"), float("nan"), float("nan")), (float("inf"), 1e30, -float("inf"), 1e30)):
        Q[pad_q], K[pad_k], V[pad_k], dO[pad_q] = query, key, value, grad
        O, lse = moba.window_forward(sh, Q, K, V, first_key=first)
        out.append((O, lse) + moba.window_backward(sh, Q, K, V, O, lse, dO, first_key=first))
    for other in out[1:]:
        for name, x, y in zip(("O", "lse", "dQ", "dK", "dV"), out[0], other):
            assert torch.equal(x, y), name
    for x, rows in zip(out[0], (pad_q, pad_q, pad_q, pad_k, pad_k)):
        assert (x[rows] == (0 if x.dim() == 4 else -float("inf"))).all()
