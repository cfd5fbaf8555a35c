"""Attention to the last W keys and its backward against the formulas in 64 bits, at the sizes and masks where
tiles and ranges end: one token, odd lengths, windows shorter and longer than a tile, shared heads, caches with
room, packed and padded batches, rows that attend nothing, infinities and NaN next to a row's pairs."""
import numpy as np
import pytest
import torch

import paper_2511_11571_amd as moba
from tests import window_reference as ref
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}


def _draw(seed, b, h, hkv, q, rows, d, dt):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
    return t(b, h, q, d), t(b, hkv, rows, d), t(b, hkv, rows, d), t(b, h, q, d)


def _check(sh, Q, K, V, dO=None, first=None):
    N = sh.kv_len
    O, lse = moba.window_forward(sh, Q, K, V, first_key=first)
    want = ref.window(Q, K[:, :, :N], V[:, :, :N], sh.window, first, sh.softmax_scale, dO)
    ref.close(O, want["O"], "O")
    ref.close(lse, want["lse"], "lse")
    if dO is not None:
        grads = moba.window_backward(sh, Q, K, V, O, lse, dO, first_key=first)
        for name, x in zip(("dQ", "dK", "dV"), grads):
            ref.close(x, want[name], name, None if name == "dQ" else N)
        return O, lse, grads
    return O, lse


def _shape(b, h, hkv, q, N, d, W, dt, rows=0, scale=0.0):
    return moba.WindowShape(b, h, q, N, d, window=W, dtype=CODE[dt], softmax_scale=scale, kv_heads=hkv, kv_rows=rows)


# batch, heads, kv heads, q_len, kv_len, window
CASES = [
    (1, 1, 1, 1, 1, 0), (1, 2, 2, 2, 2, 1), (1, 1, 1, 31, 31, 0), (2, 2, 1, 33, 33, 5), (1, 3, 1, 64, 64, 64),
    (1, 2, 2, 65, 65, 0), (1, 1, 1, 127, 127, 100), (1, 4, 2, 129, 129, 128), (2, 3, 3, 200, 200, 33),
    (1, 2, 1, 257, 257, 256), (1, 1, 1, 300, 300, 1), (1, 2, 2, 511, 511, 63), (1, 4, 1, 640, 640, 0),
    (1, 1, 1, 70, 333, 40), (1, 2, 1, 130, 500, 0), (2, 2, 2, 5, 400, 7), (1, 8, 1, 3, 129, 64),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(case, dt, d):
    b, h, hkv, q, N, W = case
    Q, K, V, dO = _draw(sum(case) + d, b, h, hkv, q, N, d, dt)
    _check(_shape(b, h, hkv, q, N, d, W, dt), Q, K, V, dO)


# enough tiles of queries, or of keys, for the kernels that work tile by tile: both of them; neither, but each on its own; with shared heads; dense; fewer
# queries than keys; queries by tiles and keys not (heads that share); the other way round (few queries)
TILES = [
    (2, 70, 70, 131, 131, 40), (2, 20, 20, 131, 131, 40), (2, 24, 6, 131, 131, 0), (2, 128, 64, 131, 131, 33), (1, 264, 264, 200, 200, 0), (1, 200, 200, 100, 300, 45),
    (1, 300, 300, 257, 257, 256), (1, 256, 16, 131, 131, 40), (1, 200, 200, 20, 300, 45), (3, 50, 50, 129, 129, 1),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", TILES, ids=str)
def test_forward_and_backward_tile_by_tile(case, dt, d):
    b, h, hkv, q, N, W = case
    Q, K, V, dO = _draw(sum(case) + d, b, h, hkv, q, N, d, dt)
    first = None
    if (q + W) % 2:                                          # half of them with sequences that start on the way
        g = torch.Generator().manual_seed(q)
        starts = torch.randint(0, 2, (b, q), generator=g).cumsum(1) * 7
        first = torch.minimum(starts.to(torch.int32), torch.arange(N - q, N, dtype=torch.int32)).cuda()
    _check(_shape(b, h, hkv, q, N, d, W, dt), Q, K, V, dO, first)


# the last few positions against a long cache: few queries, keys shared out among workgroups
TOKENS = [
    (1, 1, 1, 1, 2000, 0), (2, 4, 2, 1, 4097, 0), (1, 16, 4, 4, 3001, 0), (1, 8, 1, 7, 5000, 1000), (3, 2, 2, 16, 2500, 256),
    (1, 2, 2, 1, 9000, 256), (1, 40, 1, 1, 2049, 0), (1, 33, 1, 3, 1500, 700), (1, 1, 1, 1, 70, 70), (4, 16, 16, 1, 640, 0),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", TOKENS, ids=str)
def test_few_tokens_against_a_cache_with_room(case, dt, d):
    b, h, hkv, q, N, W = case
    rows = N + 61
    Q, K, V, _ = _draw(sum(case), b, h, hkv, q, rows, d, dt)
    K[:, :, N:], V[:, :, N:] = float("nan"), float("inf")    # rows behind the last key are not read
    sh = _shape(b, h, hkv, q, N, d, W, dt, rows)
    _check(sh, Q, K, V)
    # sequences of a padded batch that begin late, in the middle of a share or behind all keys
    first = torch.tensor([[0, N - 1, N // 2 + 3, N][(i + r) % 4] for i in range(b) for r in range(q)], dtype=torch.int32).view(b, q).cuda()
    _check(sh, Q, K, V, first=first)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv,W", [(4, 2, 96), (64, 64, 40)])
def test_packed_batch_is_each_sequence_on_its_own(h, hkv, W, dt, d):
    lens = [1, 130, 64, 0, 77, 200]
    offs = np.concatenate([[0], np.cumsum(lens)])
    N = int(offs[-1])
    lay = moba.VarlenLayout([int(x) for x in offs], 32)
    first = lay.first_key()
    want = np.repeat(offs[:-1], lens)
    assert np.array_equal(first.cpu().numpy()[0], want)
    Q, K, V, dO = _draw(3, 1, h, hkv, N, N, d, dt)
    O, lse, grads = _check(_shape(1, h, hkv, N, N, d, W, dt), Q, K, V, dO, first)
    for i, n in enumerate(lens):
        if n == 0:
            continue
        cut = lambda x: x[:, :, offs[i]:offs[i + 1]].contiguous()  # noqa: E731
        o, _, g = _check(_shape(1, h, hkv, n, n, d, W, dt), cut(Q), cut(K), cut(V), cut(dO))
        # a tile of the packed batch may hold other rows: other sums, same values but for rounding (twice the bounds)
        assert torch.allclose(o.float(), cut(O).float(), atol=2e-2 if dt == torch.bfloat16 else 1e-5)
    padded = lay.first_key(padded=True).cpu().numpy()[0]
    pad = np.asarray(lay.pad_offsets_host)
    assert np.array_equal(padded, pad[np.searchsorted(pad, np.arange(lay.padded_tokens), side="right") - 1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h,hkv,W", [(2, 1, 0), (2, 1, 50), (36, 36, 40)])
def test_rows_that_attend_nothing(dt, d, h, hkv, W):
    """A padded batch: rows of padding attend nothing, whatever they hold, and rows in no order of first keys."""
    b, N = 3, 230
    Q, K, V, dO = _draw(5, b, h, hkv, N, N, d, dt)
    first = torch.zeros((b, N), dtype=torch.int32)
    first[0, :70], first[0, 70:] = 1 << 30, 70               # padding on the left
    first[1, 100:] = N                                       # and on the right
    first[2] = torch.from_numpy(np.random.default_rng(1).integers(-300, N + 50, N).astype(np.int32))
    first = first.cuda()
    off = first > torch.arange(N, device="cuda")
    bad = off[:, None].expand(b, h, N)
    O, lse, (dQ, dK, dV) = _check(_shape(b, h, hkv, N, N, d, W, dt), Q, K, V, dO, first)
    assert (O[bad] == 0).all() and (lse[bad] == -float("inf")).all() and (dQ[bad] == 0).all()
    # the same with rubbish in those rows, and in keys that nobody attends
    Q2, dO2, K2, V2 = Q.clone(), dO.clone(), K.clone(), V.clone()
    Q2[bad], dO2[bad] = float("nan"), float("inf")
    nobody = torch.from_numpy(~ref.seen(N, N, W, first.cpu().numpy(), b).any(1)).cuda()[:, None].expand(b, hkv, N)
    assert nobody.any()
    K2[nobody], V2[nobody] = float("inf"), float("nan")
    sh = _shape(b, h, hkv, N, N, d, W, dt)
    O2, lse2 = moba.window_forward(sh, Q2, K2, V2, first_key=first)
    g2 = moba.window_backward(sh, Q2, K2, V2, O2, lse2, dO2, first_key=first)
    want = ref.window(Q2, K2, V2, W, first, dO=dO2)
    for name, x in zip(("O", "lse", "dQ", "dK", "dV"), (O2, lse2) + g2):
        ref.close(x, want[name], name)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,h,hkv,N,W", [(1, 1, 1, 1, 0), (1, 2, 1, 300, 1), (2, 20, 20, 131, 1), (2, 70, 70, 131, 1), (1, 256, 16, 131, 1)])
def test_a_single_key_gives_no_gradient_to_its_logit(b, h, hkv, N, W, d, dt):
    """The softmax of one logit is one: dQ of rows that attend one key is zero, not a rounding (the first row of every
    sequence is such a row in any window), and so is dK where the window is one key."""
    Q, K, V, dO = _draw(6, b, h, hkv, N, N, d, dt)
    _, _, (dQ, dK, dV) = _check(_shape(b, h, hkv, N, N, d, W, dt), Q, K, V, dO)
    assert not dQ.any() and not dK.any() and dV.any()
    for first in (None, torch.arange(N, dtype=torch.int32).div(7, rounding_mode="floor").mul(7).expand(b, N).contiguous().cuda()):
        _, _, (dQ, _, _) = _check(_shape(b, h, hkv, N, N, d, 40, dt), Q, K, V, dO, first)
        assert not dQ[:, :, 0].any() and (first is None or not dQ[:, :, ::7].any())
    if h <= 2:                                               # a packed batch of sequences of one
        _, _, (dQ, dK, _) = _check(_shape(b, h, hkv, N, N, d, 40, dt), Q, K, V, dO, torch.arange(N, dtype=torch.int32).expand(b, N).contiguous().cuda())
        assert not dQ.any() and not dK.any()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,N", [(33, 64), (32, 63), (40, 111), (17, 33), (5, 5)])
def test_sequences_of_one_at_the_end_of_a_cache(q, N, d, dt):
    """As above, with the rows' positions shifted against the tiles of the keys."""
    Q, K, V, dO = _draw(7, 1, 2, 2, q, N, d, dt)
    first = torch.arange(N - q, N, dtype=torch.int32).view(1, q).cuda()
    _, _, (dQ, dK, _) = _check(_shape(1, 2, 2, q, N, d, 0, dt), Q, K, V, dO, first)
    assert not dQ.any() and not dK.any()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("h,d", [(2, 64), (2, 128), (80, 64), (80, 128)])
def test_a_bad_value_reaches_the_rows_that_attend_it_and_no_other(h, d, dt, value):
    N, W, at = 300, 40, 117
    Q, K, V, dO = _draw(8, 1, h, h, N, N, d, dt)
    sh = _shape(1, h, h, N, N, d, W, dt)
    want = ref.window(Q, K, V, W, None, dO=dO)
    t = torch.arange(N)
    touched = (t >= at) & (t < at + W)
    near = (t > at - W) & (t < at + W)                        # keys that share a row with the bad one
    for which in ("K", "V"):
        K2, V2 = K.clone(), V.clone()
        (K2 if which == "K" else V2)[0, 1, at, 3] = value
        O, lse = moba.window_forward(sh, Q, K2, V2)
        grads = moba.window_backward(sh, Q, K2, V2, O, lse, dO)
        for name, x, rows in zip(("O", "lse", "dQ", "dK", "dV"), (O, lse) + grads, (touched, touched, touched, near, near)):
            value_, bound = want[name]
            keep = ~rows.numpy()
            others = [i for i in range(h) if i != 1]
            ref.close(x[:, others], (value_[:, others], bound[:, others]), name)
            ref.close(x[:, 1:2, keep], (value_[:, 1:2, keep], bound[:, 1:2, keep]), name)
        if which == "V":
            assert not torch.isfinite(O[0, 1, touched][:, 3]).any()
    # a bad query reaches its own row, and the gradients of the keys that it attends
    Q2 = Q.clone()
    Q2[0, 1, at, 3] = value
    O, lse = moba.window_forward(sh, Q2, K, V)
    dQ, dK, dV = moba.window_backward(sh, Q2, K, V, O, lse, dO)
    mine, seen = t == at, (t > at - W) & (t <= at)
    for name, x, rows in (("O", O, mine), ("dQ", dQ, mine), ("dK", dK, seen), ("dV", dV, seen)):
        value_, bound = want[name]
        keep = ~rows.numpy()
        ref.close(x[:, 1:2, keep], (value_[:, 1:2, keep], bound[:, 1:2, keep]), name)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,q,N,W", [(2, 300, 300, 100), (80, 300, 300, 100), (2, 3, 3000, 0), (130, 140, 140, 0)])
def test_nan_throughout(h, q, N, W, d, dt):
    """What a diverged model hands over: every row's own pairs are NaN, and so is everything that has some.  A sequence
    that starts at key 70 has none of them where the NaN end there."""
    Q, K, V, dO = _draw(14, 1, h, h, q, N, d, dt)
    sh = _shape(1, h, h, q, N, d, W, dt)
    nan = torch.full_like(K, float("nan"))
    O, lse = moba.window_forward(sh, Q, nan, V)
    assert torch.isnan(O).all() and torch.isnan(lse).all()
    dQ, dK, dV = moba.window_backward(sh, Q, nan, V, O, lse, dO)
    t = torch.arange(N - q, N)
    single = (t == 0) | (W == 1)
    assert torch.isnan(dQ[:, :, ~single]).all()
    seen = torch.from_numpy(ref.seen(q, N, W, None, 1)[0].any(0).copy())
    assert torch.isnan(dV[:, :, seen]).all() and torch.isnan(dK[:, :, seen]).all()
    assert not dV[:, :, ~seen].any() and not dK[:, :, ~seen].any()
    if q == N:
        start = torch.full((1, q), 70, dtype=torch.int32)
        start[:, :70] = 0
        K2 = K.clone()
        K2[:, :, :70] = float("nan")
        first = start.cuda()
        O, lse = moba.window_forward(sh, Q, K2, V, first_key=first)
        grads = moba.window_backward(sh, Q, K2, V, O, lse, dO, first_key=first)
        want = ref.window(Q, K, V, W, first, dO=dO)
        for name, x in zip(("O", "lse", "dQ", "dK", "dV"), (O, lse) + grads):
            ref.close(x[:, :, 70:], tuple(w[:, :, 70:] for w in want[name]), name)
            assert torch.isnan(x[:, :, 1:70]).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.3, 1e-4])
@pytest.mark.parametrize("h,W", [(2, 128), (70, 50)])
def test_scales_and_large_logits(h, W, dt, scale):
    """Logits of tens to hundreds: the running maximum moves, most weights vanish."""
    Q, K, V, dO = _draw(9, 1, h, h, 260, 260, 64, dt)
    K[:, :, 40] *= 6
    K[:, :, 200] *= 9
    _check(_shape(1, h, h, 260, 260, 64, W, dt, scale=scale), Q, K, V, dO)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gradients_against_differences(dt):
    """d/de of sum(O * dO) along random directions, taken in 64 bits by central differences of the formula."""
    b, h, hkv, N, d, W = 1, 4, 2, 90, 64, 37
    Q, K, V, dO = _draw(10, b, h, hkv, N, N, d, dt)
    sh = _shape(b, h, hkv, N, N, d, W, dt)
    O, lse = moba.window_forward(sh, Q, K, V)
    grads = moba.window_backward(sh, Q, K, V, O, lse, dO)
    on = torch.from_numpy(ref.seen(N, N, W, None, b)[0].copy())

    def f(x):
        q, k, v = x[0], x[1].repeat_interleave(h // hkv, 1), x[2].repeat_interleave(h // hkv, 1)
        s = (q @ k.transpose(-1, -2) / 8.0).masked_fill(~on, -float("inf"))
        return float(((torch.softmax(s, -1) @ v) * dO.cpu().double()).sum())

    x = [t.cpu().double() for t in (Q, K, V)]
    want = ref.window(Q, K, V, W, None, dO=dO)
    g = torch.Generator().manual_seed(11)
    for i, name in enumerate(("dQ", "dK", "dV")):
        v = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
        step = 1e-4
        diff = (f(x[:i] + [x[i] + step * v] + x[i + 1:]) - f(x[:i] + [x[i] - step * v] + x[i + 1:])) / (2 * step)
        got = float((grads[i].cpu().double() * v).sum())
        # the elements' bounds, and the differences' own error (third derivatives times step^2)
        assert abs(got - diff) <= float((want[name][1] * v.abs().numpy()).sum()) + 1e-5 * float(v.norm())


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,hkv,W", [(4, 2, 100), (90, 90, 40)])
def test_nothing_outside_the_buffers_is_written(h, hkv, W, d, dt):
    b, N = 1, 210
    rows, guard = 240, 4096
    Q, K, V, dO = _draw(12, b, h, hkv, N, rows, d, dt)
    sh = _shape(b, h, hkv, N, N, d, W, dt, rows)

    def room(shape, dtype):
        n = int(np.prod(shape)) * torch.finfo(dtype).bits // 8
        raw = torch.full((n + 2 * guard,), 0xa5, dtype=torch.uint8, device="cuda")
        return raw, raw[guard:guard + n].view(dtype).view(shape)

    bufs = {n: room(s, t) for n, s, t in (("O", Q.shape, Q.dtype), ("lse", Q.shape[:3], torch.float32), ("dQ", Q.shape, Q.dtype),
                                          ("dK", K.shape, Q.dtype), ("dV", K.shape, Q.dtype))}
    need = moba.window_workspace_bytes(sh)
    ws = torch.full((max(need) + 2 * guard,), 0xa5, dtype=torch.uint8, device="cuda")
    moba.window_forward(sh, Q, K, V, ws=ws[guard:guard + need[0]], O=bufs["O"][1], lse=bufs["lse"][1])
    moba.window_backward(sh, Q, K, V, bufs["O"][1], bufs["lse"][1], dO, ws=ws[guard:guard + need[1]],
                         out=tuple(bufs[n][1] for n in ("dQ", "dK", "dV")))
    torch.cuda.synchronize()
    for name, (raw, _) in bufs.items():
        assert (raw[:guard] == 0xa5).all() and (raw[-guard:] == 0xa5).all(), name
    assert (ws[:guard] == 0xa5).all() and (ws[-guard - max(need) + need[1]:] == 0xa5).all()
    for n in ("dK", "dV"):                                   # rows behind the last key
        assert (bufs[n][0][guard:-guard].view(hkv, rows, -1)[:, N:] == 0xa5).all()


def test_streams_graphs_and_repeats():
    """A captured pass replayed after eager work of the same shapes, and on another stream, gives the same bits."""
    shapes = [(_shape(1, 4, 2, 400, 400, 64, 90, torch.bfloat16), True), (_shape(1, 8, 2, 2, 3000, 128, 0, torch.bfloat16), False),
              (_shape(1, 48, 48, 400, 400, 128, 40, torch.bfloat16), True)]
    for sh, train in shapes:
        q, N = sh.q_len, sh.kv_len
        Q, K, V, dO = _draw(13, 1, sh.heads, sh.hkv, q, N, sh.head_dim, torch.bfloat16)

        def step(ws=None):
            O, lse = moba.window_forward(sh, Q, K, V, ws=ws)
            return (O, lse) + (moba.window_backward(sh, Q, K, V, O, lse, dO, ws=ws) if train else ())

        want = [x.clone() for x in step()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            there = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, there))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        keep = Q.clone()
        for i in range(3):
            Q.copy_(keep if i != 1 else keep.roll(1, -1))
            graph.replay()
            torch.cuda.synchronize()
            now = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, now))
            assert i == 1 or all(torch.equal(a, b) for a, b in zip(held, want))


def test_offsets_beyond_32_bits():
    """A cache of 2^24 rows in fp32: the last keys lie 8 GB behind the first, those of the second head 17 GB."""
    h, N, d, W, q = 2, 1 << 24, 128, 200, 3
    K, V = (torch.empty((1, h, N, d), device="cuda") for _ in range(2))
    near = 256
    g = torch.Generator().manual_seed(17)
    for t in (K, V):
        t[:, :, -near:] = torch.randn((1, h, near, d), generator=g).cuda()
        t[:, :, -near - W:-near] = 0.0
    Q, dO = (torch.randn((1, h, q, d), generator=g).cuda() for _ in range(2))
    cut = [t[:, :, -near:].contiguous() for t in (K, V)]
    sh = _shape(1, h, h, q, N, d, W, torch.float32)
    O, lse = moba.window_forward(sh, Q, K, V)
    want = ref.window(Q, *cut, W, None, dO=dO)
    ref.close(O, want["O"], "O")
    ref.close(lse, want["lse"], "lse")
    dQ, dK, dV = moba.window_backward(sh, Q, K, V, O, lse, dO)
    ref.close(dQ, want["dQ"], "dQ")
    for name, x in (("dK", dK), ("dV", dV)):
        ref.close(x[:, :, -near:].contiguous(), want[name], name)
        assert not x[:, :, :-near].any()                     # keys that no row attends
    del K, V, dK, dV
    torch.cuda.empty_cache()
