"""Rotary positions and their gradient against the formula in 64 bits.  A result is one rounding to the I/O type, h,
and a cosine and a sine that are off by c: 2^-16 for bf16 (the chip's own), 2^-21 for fp32 (32-bit products included)."""
import numpy as np
import pytest
import torch

import paper_2511_11571_amd as moba
from tests import window_reference as ref
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}
TRIG = {torch.float32: 2.0 ** -21, torch.bfloat16: 2.0 ** -16}


def _draw(seed, shape, dt):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()


def _close(got, x, sh, pos, back=False):
    want, mag = ref.rope(x, pos, sh.rot_dim or sh.head_dim, sh.interleaved, ref.rope_frequencies(sh), np.float32(sh.amplitude), back)
    a = got.detach().cpu().double().numpy()
    dt = x.dtype
    bound = ref.half_step(dt) * np.abs(want) + (1 + ref.half_step(dt)) * TRIG[dt] * mag
    rot = sh.rot_dim or sh.head_dim
    bound[..., rot:] = 0.0                                    # copied
    off = np.abs(a - want)
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert np.all(off <= bound), f"{worst}: {a[worst]} is not {want[worst]}"


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,h,hkv,N,d,rot", [(1, 1, 1, 1, 64, 0), (2, 3, 1, 37, 64, 48), (1, 4, 4, 130, 128, 0), (1, 2, 2, 5, 128, 96),
                                             (3, 2, 1, 9, 64, 20), (1, 5, 1, 33, 64, 2), (1, 1, 1, 600, 128, 126), (1, 8, 2, 300, 64, 32)])
def test_layouts_and_parts_of_the_head(b, h, hkv, N, d, rot, dt, interleaved, back):
    sh = moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt], rot_dim=rot, interleaved=interleaved, position0=1000, amplitude=1.25)
    Q, K = _draw(N, (b, h, N, d), dt), _draw(N + 1, (b, hkv, N, d), dt)
    f = moba.rope_backward if back else moba.rope
    q, k = f(sh, Q, K)
    pos = np.broadcast_to(1000.0 + np.arange(N), (b, N))
    _close(q, Q, sh, pos, back)
    _close(k, K, sh, pos, back)
    alone, none = f(sh, Q)
    assert none is None and torch.equal(alone, q)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("theta,factor,orig,low,high", [(1e4, 1.0, 0, 1, 32), (5e5, 8.0, 0, 1, 32), (5e5, 8.0, 8192, 1, 32), (1e6, 40.0, 4096, 1, 4),
                                                        (1e4, 0.5, 2048, 0.5, 2)])
def test_scaled_frequencies_at_far_positions(theta, factor, orig, low, high, dt):
    b, h, N, d = 2, 2, 12, 128
    sh = moba.RopeShape(b, h, N, d, dtype=CODE[dt], theta=theta, scale_factor=factor, orig_len=orig, band_low=low, band_high=high)
    pos = torch.tensor([[0, 1, 2, 4095, 131071, 1 << 20, 10 ** 6, 16777217, 2 ** 31 - 1, -1, -131072, -2 ** 31],
                        list(range(99990, 100002))], dtype=torch.int32)
    Q, K = _draw(1, (b, h, N, d), dt), _draw(2, (b, h, N, d), dt)
    for back, f in ((False, moba.rope), (True, moba.rope_backward)):
        q, k = f(sh, Q, K, pos.cuda())
        _close(q, Q, sh, pos.double().numpy(), back)
        _close(k, K, sh, pos.double().numpy(), back)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_in_place_and_into_a_cache(dt):
    b, h, hkv, N, d, rows, at = 2, 4, 2, 3, 64, 50, 17
    sh = moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt], rot_dim=32, position0=at, k_out_rows=rows)
    Q, K = _draw(3, (b, h, N, d), dt), _draw(4, (b, hkv, N, d), dt)
    want_q, want_k = moba.rope(moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt], rot_dim=32, position0=at), Q, K)
    cache = torch.full((b, hkv, rows, d), 7.0, dtype=dt, device="cuda")
    q, k = moba.rope(sh, Q, K, out=(None, cache[:, :, at:at + N]))
    assert torch.equal(q, want_q) and torch.equal(cache[:, :, at:at + N], want_k)
    cache[:, :, at:at + N] = 7.0
    assert (cache == 7.0).all()                               # nothing else was written
    same = moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt], rot_dim=32, position0=at)
    q2, k2 = Q.clone(), K.clone()
    moba.rope(same, q2, k2, out=(q2, k2))
    assert torch.equal(q2, want_q) and torch.equal(k2, want_k)
    # tensors that start at any element
    raw = torch.zeros(Q.numel() + 1, dtype=dt, device="cuda")[1:].view(Q.shape)
    raw.copy_(Q)
    odd, _ = moba.rope(same, raw)
    assert torch.equal(odd, want_q)


def test_there_and_back_and_many_heads():
    """The gradient of a turn is the turn back: the two in a row give the input (amplitude 1; two roundings and four
    sines), over a grid that splits the heads."""
    dt = torch.float32
    sh = moba.RopeShape(1, 48, 4099, 64, kv_heads=3, dtype=CODE[dt])
    Q, K = _draw(5, (1, 48, 4099, 64), dt), _draw(6, (1, 3, 4099, 64), dt)
    q, k = moba.rope_backward(sh, *moba.rope(sh, Q, K))
    for got, x in ((q, Q), (k, K)):
        mag = x.abs()[..., :32] + x.abs()[..., 32:]
        assert ((got - x).abs() <= 8 * 2.0 ** -21 * torch.cat((mag, mag), -1)).all()


def test_a_hybrid_models_layer_runs_together():
    """Rotary positions, window attention and both backwards as a training step, against the formulas end to end, and
    a serving step that goes on from the step's keys: its token's output is that of the longer sequence."""
    b, h, hkv, N, d, W, dt = 1, 4, 2, 200, 64, 64, torch.float32
    Q, K, V, dO = (_draw(i, (b, x, N, d), dt) for i, x in ((1, h), (2, hkv), (3, hkv), (4, h)))
    rs = moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt])
    ws = moba.WindowShape(b, h, N, N, d, window=W, dtype=CODE[dt], kv_heads=hkv)
    q, k = moba.rope(rs, Q, K)
    O, lse = moba.window_forward(ws, q, k, V)
    dq, dk, dV = moba.window_backward(ws, q, k, V, O, lse, dO)
    dQ, dK = moba.rope_backward(rs, dq, dk)
    on = torch.from_numpy(ref.seen(N, N, W, None, b)[0].copy())
    x = [t.cpu().double().requires_grad_() for t in (Q, K, V)]
    ang = torch.arange(N).double()[:, None] * torch.tensor(ref.rope_frequencies(rs), dtype=torch.float64)

    def turned(t):
        a, c = t[..., :32], t[..., 32:]
        return torch.cat((a * ang.cos() - c * ang.sin(), c * ang.cos() + a * ang.sin()), -1)

    s = turned(x[0]) @ turned(x[1]).repeat_interleave(2, 1).transpose(-1, -2) / 8.0
    o = torch.softmax(s.masked_fill(~on, -float("inf")), -1) @ x[2].repeat_interleave(2, 1)
    o.backward(dO.cpu().double())
    # fp32 throughout: the bounds of the stages come to some 1e-5 for values of this size
    for got, want in ((O, o), (dQ, x[0].grad), (dK, x[1].grad), (dV, x[2].grad)):
        assert (got.cpu().double() - want).abs().max() < 1e-4
    # the last position once more, as a serving step: its key goes into the cache, the token attends it
    cache_k, cache_v = k.new_zeros(b, hkv, N + 8, d), k.new_zeros(b, hkv, N + 8, d)
    cache_k[:, :, :N - 1], cache_v[:, :, :N] = k[:, :, :N - 1], V
    step = moba.RopeShape(b, h, 1, d, kv_heads=hkv, dtype=CODE[dt], position0=N - 1, k_out_rows=N + 8)
    qt, _ = moba.rope(step, Q[:, :, N - 1:].contiguous(), K[:, :, N - 1:].contiguous(), out=(None, cache_k[:, :, N - 1:N]))
    ot, lt = moba.window_forward(moba.WindowShape(b, h, 1, N, d, window=W, dtype=CODE[dt], kv_heads=hkv, kv_rows=N + 8), qt, cache_k, cache_v)
    assert (ot[:, :, 0] - O[:, :, -1]).abs().max() < 1e-5 and (lt[:, :, 0] - lse[:, :, -1]).abs().max() < 1e-5


def test_offsets_beyond_32_bits():
    """2^24 rows of fp32, 8 GB, in place: the last rows as a call on them alone."""
    n, d = 1 << 24, 128
    x = torch.empty((1, 1, n, d), device="cuda")
    x[:, :, :64], x[:, :, -64:] = _draw(7, (1, 1, 64, d), torch.float32), _draw(8, (1, 1, 64, d), torch.float32)
    ends = x[:, :, :64].clone(), x[:, :, -64:].clone()
    moba.rope(moba.RopeShape(1, 1, n, d, dtype=binding.F32), x, out=(x, None))
    for got, a, at in ((x[:, :, :64], ends[0], 0), (x[:, :, -64:], ends[1], n - 64)):
        want, _ = moba.rope(moba.RopeShape(1, 1, 64, d, dtype=binding.F32, position0=at), a)
        assert torch.equal(got, want)
    del x
    torch.cuda.empty_cache()
