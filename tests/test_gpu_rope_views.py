"""Rotary positions of stretches of larger tensors, to stretches of others; captured and replayed; and the first keys of packed
batches with empty sequences and rows behind the last one."""
import ctypes

import pytest
import torch

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

pytestmark = pytest.mark.gpu

CODE = {torch.float32: binding.F32, torch.bfloat16: binding.BF16}


def _draw(seed, shape, dt):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rot", [0, 20, 48])
@pytest.mark.parametrize("rows", [dict(q_rows=40, k_rows=64, q_out_rows=31, k_out_rows=99), dict(k_rows=50), dict(q_out_rows=77), dict(q_rows=33, q_out_rows=33)])
def test_from_and_to_parts_of_larger_tensors(rows, rot, dt, interleaved):
    b, h, hkv, N, d = 2, 4, 2, 29, 64
    base = dict(kv_heads=hkv, dtype=CODE[dt], rot_dim=rot, interleaved=interleaved, position0=500)
    Q, K = _draw(1, (b, h, N, d), dt), _draw(2, (b, hkv, N, d), dt)
    positions = torch.randint(0, 100000, (b, N), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    for pos in (None, positions):
        for f in (moba.rope, moba.rope_backward):
            want_q, want_k = f(moba.RopeShape(b, h, N, d, **base), Q, K, pos)

            def room(x, n, fill):                            # x's rows as a stretch that begins at row 2, or at 0 if there is no room
                n = n or N
                t = torch.full((b, x.shape[1], n, d), fill, dtype=dt, device="cuda")
                at = min(2, n - N)
                return t, t[:, :, at:at + N], at

            big_q, q, _ = room(Q, rows.get("q_rows"), 3.0)
            big_k, k, _ = room(K, rows.get("k_rows"), 3.0)
            q.copy_(Q)
            k.copy_(K)
            to_q, qo, aq = room(Q, rows.get("q_out_rows"), 9.0)
            to_k, ko, ak = room(K, rows.get("k_out_rows"), 9.0)
            f(moba.RopeShape(b, h, N, d, **base, **rows), q, k, pos, out=(qo, ko))
            assert torch.equal(qo, want_q) and torch.equal(ko, want_k)
            assert torch.equal(q, Q) and torch.equal(k, K)
            qo.fill_(9.0)
            ko.fill_(9.0)
            assert (to_q == 9.0).all() and (to_k == 9.0).all()           # nothing else was written
            # in place, where the rows of a slice are as many
            same = dict(rows, q_out_rows=rows.get("q_rows", 0), k_out_rows=rows.get("k_rows", 0))
            f(moba.RopeShape(b, h, N, d, **base, **same), q, k, pos, out=(q, k))
            assert torch.equal(q, want_q) and torch.equal(k, want_k)
            q.fill_(3.0)
            k.fill_(3.0)
            assert (big_q == 3.0).all() and (big_k == 3.0).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_replayed_and_on_another_stream(dt):
    b, h, hkv, N, d = 2, 6, 3, 300, 128
    sh = moba.RopeShape(b, h, N, d, kv_heads=hkv, dtype=CODE[dt], theta=5e5, scale_factor=8.0, orig_len=8192)
    Q, K = _draw(4, (b, h, N, d), dt), _draw(5, (b, hkv, N, d), dt)
    pos = torch.arange(N, dtype=torch.int32).expand(b, N).contiguous().cuda()
    want = [x.clone() for x in moba.rope(sh, Q, K, pos)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = moba.rope(sh, Q, K, pos)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, there))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = moba.rope(sh, Q, K, pos)
    for i in range(4):
        pos += 1000
        graph.replay()
        now = moba.rope(sh, Q, K, pos)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(held, now)) and not torch.equal(now[0], want[0])


@pytest.mark.parametrize("lens", [[5], [0, 5, 0, 0, 3, 0], [1] * 300, [257, 0, 256, 1, 511], [0, 0, 7]])
def test_first_keys_of_packed_batches(lens):
    offs = [0]
    for n in lens:
        offs.append(offs[-1] + n)
    dev = torch.tensor(offs, dtype=torch.int32, device="cuda")
    more = offs[-1] + 300                                    # rows behind the last sequence stay as they are
    out = torch.full((more,), -7, dtype=torch.int32, device="cuda")
    f = moba.lib().moba_varlen_first_key
    st = f(len(lens), ctypes.c_void_p(dev.data_ptr()), more, ctypes.c_void_p(out.data_ptr()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    want = [o for o, n in zip(offs, lens) for _ in range(n)] + [-7] * 300
    assert st == 0 and out.tolist() == want
    out.fill_(-7)
    f(len(lens), ctypes.c_void_p(dev.data_ptr()), 3, ctypes.c_void_p(out.data_ptr()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert out.tolist() == want[:3] + [-7] * (more - 3)
