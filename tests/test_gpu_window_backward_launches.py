"""Backward of short calls: sizes on either side of the choice between one launch for both directions and two."""
import pytest
import torch

import paper_2511_11571_amd as moba
from tests import window_reference as ref
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv,N", [(5, 5, 700), (8, 8, 600), (16, 16, 520), (8, 2, 400)])
@pytest.mark.parametrize("share", [0, 3])                     # dense, or windows of a third of the keys
def test_one_launch_or_two(share, h, hkv, N, dt, d):
    g = torch.Generator().manual_seed(h + N + d)
    t = lambda n: torch.randn((1, n, N, d), generator=g).to(dt).cuda()  # noqa: E731
    Q, K, V, dO = t(h), t(hkv), t(hkv), t(h)
    W = N // share if share else 0
    sh = moba.WindowShape(1, h, N, N, d, window=W, dtype=CODE[dt], kv_heads=hkv)
    O, lse = moba.window_forward(sh, Q, K, V)
    grads = moba.window_backward(sh, Q, K, V, O, lse, dO)
    want = ref.window(Q, K, V, W, None, dO=dO)
    for name, x in zip(("O", "lse", "dQ", "dK", "dV"), (O, lse) + grads):
        ref.close(x, want[name], name)
