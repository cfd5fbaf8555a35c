"""Window attention where workgroups share the keys of rows and a second kernel joins their parts, with many groups of rows at
different positions: short dense calls, shared heads that do not divide a group, queries at the end of a cache, with and
without first keys; and the bounds of the workspace that the parts are kept in."""
import numpy as np
import pytest
import torch

import paper_2511_11571_amd as moba
from tests import window_reference as ref
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}

# batch, heads, kv heads, q_len, kv_len, window
SHARED = [(1, 2, 2, 2048, 2048, 0), (1, 1, 1, 1101, 1101, 0), (1, 3, 1, 700, 2000, 0), (1, 5, 1, 300, 1900, 1024), (2, 3, 1, 333, 2100, 1500),
          (1, 1, 1, 2100, 2100, 1100), (1, 40, 1, 33, 1500, 0)]


def _shape(case, d, dt, rows=0):
    b, h, hkv, q, N, W = case
    return moba.WindowShape(b, h, q, N, d, window=W, dtype=CODE[dt], kv_heads=hkv, kv_rows=rows)


def _draw(case, d, dt, rows=0):
    b, h, hkv, q, N, _ = case
    g = torch.Generator().manual_seed(sum(case) + d)
    t = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
    return t(b, h, q, d), t(b, hkv, rows or N, d), t(b, hkv, rows or N, d)


def _firsts(case):
    """No first keys; sequences of very different lengths; rows in no order, some of which attend nothing."""
    b, _, _, q, N, _ = case
    rng = np.random.default_rng(q)
    t = np.arange(N - q, N)
    cuts = np.sort(rng.choice(N, 6, replace=False))
    packed = np.array([max([0] + [int(c) for c in cuts if c <= x]) for x in t])
    loose = rng.integers(-N, N + 200, (b, q))
    return [None] + [torch.from_numpy(np.broadcast_to(f, (b, q)).astype(np.int32).copy()).cuda() for f in (packed, loose)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", SHARED, ids=str)
def test_shared_keys_of_many_groups(case, dt, d):
    sh = _shape(case, d, dt)
    assert moba.window_workspace_bytes(sh)[0] > 0            # (the keys are shared)
    Q, K, V = _draw(case, d, dt)
    for first in _firsts(case):
        O, lse = moba.window_forward(sh, Q, K, V, first_key=first)
        want = ref.window(Q, K, V, sh.window, first)
        ref.close(O, want["O"], "O")
        ref.close(lse, want["lse"], "lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", [(1, 3, 1, 700, 2000, 0), (1, 16, 4, 4, 3001, 0), (1, 40, 1, 33, 1500, 0)], ids=str)
def test_workspaces_of_any_content_and_nothing_beyond(case, dt, d):
    """The workspace may hold anything; nothing outside it, O and lse is written, and rows of K and V behind the last key,
    NaN here, are not read."""
    b, h, hkv, q, N, _ = case
    rows, guard = N + 45, 4096
    sh = _shape(case, d, dt, rows)
    need = moba.window_workspace_bytes(sh)[0]
    assert need > 0
    Q, K, V = _draw(case, d, dt, rows)
    K[:, :, N:], V[:, :, N:] = float("nan"), float("nan")
    out = []
    for fill in (0x00, 0xff, 0x7f):                          # (0xffffffff is a NaN as a float, 0x7f7f7f7f about 3.4e38)
        raw = torch.full((need + 2 * guard,), 0xa5, dtype=torch.uint8, device="cuda")
        raw[guard:guard + need] = fill
        n = Q.numel() * Q.element_size()
        o = torch.full((n + 2 * guard,), 0xa5, dtype=torch.uint8, device="cuda")
        s = torch.full((4 * b * h * q + 2 * guard,), 0xa5, dtype=torch.uint8, device="cuda")
        O, lse = o[guard:guard + n].view(dt).view(Q.shape), s[guard:-guard].view(torch.float32).view(b, h, q)
        moba.window_forward(sh, Q, K, V, ws=raw[guard:guard + need], O=O, lse=lse)
        torch.cuda.synchronize()
        for x in (raw, o, s):
            assert (x[:guard] == 0xa5).all() and (x[-guard:] == 0xa5).all()
        out.append((O.clone(), lse.clone()))
    want = ref.window(Q, K[:, :, :N], V[:, :, :N], sh.window, None)
    ref.close(out[0][0], want["O"], "O")
    ref.close(out[0][1], want["lse"], "lse")
    for O, lse in out[1:]:
        assert torch.equal(O, out[0][0]) and torch.equal(lse, out[0][1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_bad_value_in_one_share(value, dt, d):
    """It reaches the rows that attend it and no other, and those through the join as well."""
    case = (1, 2, 1, 600, 2000, 0)
    sh = _shape(case, d, dt)
    assert moba.window_workspace_bytes(sh)[0] > 0
    Q, K, V = _draw(case, d, dt)
    first = torch.zeros((1, 600), dtype=torch.int32)
    first[0, 300:] = 1200                                    # the bad key lies before these rows' sequence
    want = ref.window(Q, K, V, 0, first)
    for which in ("K", "V"):
        K2, V2 = K.clone(), V.clone()
        (K2 if which == "K" else V2)[0, 0, 1100, 5] = value
        O, lse = moba.window_forward(sh, Q, K2, V2, first_key=first.cuda())
        keep = slice(300, 600)
        ref.close(O[:, :, keep], tuple(w[:, :, keep] for w in want["O"]), "O")
        ref.close(lse[:, :, keep], tuple(w[:, :, keep] for w in want["lse"]), "lse")
        if which == "V":
            assert not torch.isfinite(O[:, :, :300, 5]).any()
            other = [c for c in range(d) if c != 5]
            ref.close(O[:, :, :300][..., other], tuple(w[:, :, :300][..., other] for w in want["O"]), "O")
        elif value != value:
            assert torch.isnan(O[:, :, :300]).all() and torch.isnan(lse[:, :, :300]).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", [(1, 2, 2, 260, 260, 128), (1, 70, 70, 260, 260, 50), (1, 3, 1, 500, 1600, 0), (1, 4, 4, 1, 3000, 0)], ids=str)
def test_large_logits_at_d_128(case, dt):
    """Logits of tens to hundreds: the running maximum moves, within a walk and from share to share."""
    b, h, hkv, q, N, W = case
    Q, K, V = _draw(case, 128, dt)
    K[:, :, 40] *= 6
    K[:, :, 200] *= 9
    K[:, :, N - 70] *= 12
    for scale in (0.3, 1e-4):
        sh = moba.WindowShape(b, h, q, N, 128, window=W, dtype=CODE[dt], kv_heads=hkv, softmax_scale=scale)
        O, lse = moba.window_forward(sh, Q, K, V)
        want = ref.window(Q, K, V, W, None, scale)
        ref.close(O, want["O"], "O")
        ref.close(lse, want["lse"], "lse")


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_graphs_with_a_workspace_of_their_own(dt):
    """Two captured steps and eager ones by turns, training calls and a few tokens with shared keys: the same bits each time."""
    cases = [((1, 4, 2, 400, 400, 90), 64, True), ((1, 2, 2, 1200, 1200, 0), 128, True), ((1, 8, 2, 2, 3000, 0), 64, False), ((1, 48, 48, 400, 400, 40), 128, True)]
    for case, d, train in cases:
        sh = _shape(case, d, dt)
        fwd, bwd = moba.window_workspace_bytes(sh)
        Q, K, V = _draw(case, d, dt)
        dO = Q.flip(-1).contiguous()
        first = torch.zeros((case[0], case[3]), dtype=torch.int32, device="cuda")

        def step(ws):
            O, lse = moba.window_forward(sh, Q, K, V, first_key=first, ws=ws)
            return (O, lse) + (moba.window_backward(sh, Q, K, V, O, lse, dO, first_key=first, ws=ws) if train else ())

        spaces = [torch.empty(max(fwd, bwd, 256), dtype=torch.uint8, device="cuda") for _ in range(3)]
        want = [x.clone() for x in step(spaces[0])]
        graphs = []
        for ws in spaces[1:]:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held = step(ws)
            graphs.append((graph, held))
        keep = Q.clone()
        for i in range(4):
            Q.copy_(keep.roll(i % 2, -1))
            for graph, _ in graphs:
                graph.replay()
            now = step(spaces[0])
            torch.cuda.synchronize()
            for _, held in graphs:
                assert all(torch.equal(a, b) for a, b in zip(held, now))
            assert i % 2 == 1 or all(torch.equal(a, b) for a, b in zip(now, want))
