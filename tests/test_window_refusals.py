"""Refusals of the window-attention and rotary calls, one fault to a call: every tensor has an address of its own and
everything but the fault is in order, so that a check that is missing shows.  Nothing is launched: the window calls are made
with a workspace that is too small, which they notice after the shape and the pointers, and a rotary call that is let through
finds no device."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
no_device = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="a call that is not refused would be launched at addresses that hold nothing")


@pytest.fixture(scope="module")
def lib():
    return moba.lib()


def _at(i):
    return 4096 * (i + 1)


def _call(f, shape, ptrs, *rest):
    return f(shape if shape is None else ctypes.byref(shape.c()), *[ctypes.c_void_p(p) for p in ptrs], *rest, None)


def _window(**kw):
    base = dict(batch=1, heads=4, q_len=1, kv_len=200000, head_dim=64, window=0, kv_heads=2)       # (a forward that takes a workspace)
    base.update(kw)
    return moba.WindowShape(**base)


FORWARD = ("Q", "K", "V", "first_key", "O", "lse", "ws")
BACKWARD = ("Q", "K", "V", "O", "lse", "dO", "first_key", "dQ", "dK", "dV", "ws")


def _window_calls(lib):
    return (("forward", lib.moba_window_forward, FORWARD), ("backward", lib.moba_window_backward, BACKWARD))


def test_a_call_in_order_gets_as_far_as_its_workspace(lib):
    need = moba.window_workspace_bytes(_window())
    assert min(need) > 256
    for i, (_, f, names) in enumerate(_window_calls(lib)):
        ptrs = [_at(j) for j in range(len(names))]
        assert _call(f, _window(), ptrs, ctypes.c_size_t(need[i] - 1)) == EWORKSPACE
        ptrs[names.index("ws")] = None
        assert _call(f, _window(), ptrs, ctypes.c_size_t(need[i])) == EWORKSPACE


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), EINVAL), (dict(batch=-1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=3), EINVAL), (dict(kv_heads=-1), EINVAL),
    (dict(q_len=0), EINVAL), (dict(q_len=200001), EINVAL), (dict(window=-1), EINVAL), (dict(kv_rows=199999), EINVAL), (dict(kv_rows=-5), EINVAL),
    (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(softmax_scale=float("nan")), EINVAL), (dict(softmax_scale=float("inf")), EINVAL),
    (dict(softmax_scale=-float("inf")), EINVAL), (dict(head_dim=0), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(head_dim=256), EUNSUPPORTED),
    (dict(kv_len=(1 << 24) + 1), EUNSUPPORTED), (dict(kv_rows=(1 << 24) + 1), EUNSUPPORTED), (dict(batch=16384), EUNSUPPORTED)], ids=str)
def test_window_shapes(lib, kw, status):
    for _, f, names in _window_calls(lib):
        assert _call(f, _window(**kw), [_at(j) for j in range(len(names))], ctypes.c_size_t(16)) == status
    with pytest.raises(moba.MobaError):
        moba.window_workspace_bytes(_window(**kw))


def test_window_workspace_pointers(lib):
    sh, a, b = _window().c(), ctypes.c_size_t(0), ctypes.c_size_t(0)
    f = lib.moba_window_workspace
    assert f(ctypes.byref(sh), ctypes.byref(a), ctypes.byref(b)) == 0 and a.value > 0 and b.value > 0
    assert f(ctypes.byref(sh), None, ctypes.byref(b)) == EINVAL and f(ctypes.byref(sh), ctypes.byref(a), None) == EINVAL


def test_window_pointers(lib):
    for call, f, names in _window_calls(lib):
        assert _call(f, None, [_at(j) for j in range(len(names))], ctypes.c_size_t(16)) == EINVAL
        for i, name in enumerate(names):
            for bad in ([None] if name not in ("first_key", "ws") else []) + [_at(i) + (2 if name in ("lse", "first_key") else 8)]:
                ptrs = [_at(j) for j in range(len(names))]
                ptrs[i] = bad
                assert _call(f, _window(), ptrs, ctypes.c_size_t(16)) == EINVAL, (call, name, bad)
        for i, name in enumerate(names):                     # the boundaries that they may start on
            ptrs = [_at(j) for j in range(len(names))]
            ptrs[i] += 4 if name in ("lse", "first_key") else 16
            assert _call(f, _window(), ptrs, ctypes.c_size_t(16)) == EWORKSPACE, (call, name)
        ptrs = [_at(j) for j in range(len(names))]
        ptrs[names.index("first_key")] = None
        assert _call(f, _window(), ptrs, ctypes.c_size_t(16)) == EWORKSPACE, call


def _rope(**kw):
    base = dict(batch=2, heads=4, seqlen=30, head_dim=64, kv_heads=2)
    base.update(kw)
    return moba.RopeShape(**base)


def _rope_calls(lib):
    return (lib.moba_rope, lib.moba_rope_backward)


ROPE = [_at(j) for j in range(5)]                             # Q K positions Q_out K_out


@no_device
def test_rotary_calls_in_order_get_as_far_as_the_device(lib):
    for f in _rope_calls(lib):
        for kw in (dict(), dict(dtype=binding.F32), dict(rot_dim=20, interleaved=True), dict(q_rows=40, k_rows=31, q_out_rows=30, k_out_rows=99),
                   dict(theta=5e5, scale_factor=8.0, orig_len=8192, amplitude=1.2), dict(position0=1 << 31), dict(position0=-(1 << 31))):
            assert _call(f, _rope(**kw), ROPE) not in (0, EINVAL, EUNSUPPORTED), kw
        for ptrs in ([ROPE[0], None, None, ROPE[3], None], ROPE[:2] + [None] + ROPE[:2]):      # queries alone; in place
            assert _call(f, _rope(), ptrs) not in (0, EINVAL, EUNSUPPORTED)


@no_device
@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), EINVAL), (dict(heads=-1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=-1), EINVAL), (dict(seqlen=0), EINVAL), (dict(dtype=3), EINVAL),
    (dict(head_dim=0), EINVAL), (dict(rot_dim=3), EINVAL), (dict(rot_dim=66), EINVAL), (dict(rot_dim=-2), EINVAL), (dict(interleaved=2), EINVAL),
    (dict(theta=0.0), EINVAL), (dict(theta=-1.0), EINVAL), (dict(theta=float("nan")), EINVAL), (dict(theta=float("inf")), EINVAL),
    (dict(scale_factor=0.0), EINVAL), (dict(scale_factor=float("nan")), EINVAL), (dict(scale_factor=float("inf")), EINVAL), (dict(orig_len=-1.0), EINVAL),
    (dict(orig_len=float("nan")), EINVAL), (dict(orig_len=float("inf")), EINVAL), (dict(orig_len=8192, band_low=4.0, band_high=4.0), EINVAL),
    (dict(orig_len=8192, band_low=float("nan")), EINVAL), (dict(orig_len=8192, band_low=-float("inf")), EINVAL), (dict(orig_len=8192, band_high=float("inf")), EINVAL),
    (dict(amplitude=float("nan")), EINVAL), (dict(amplitude=float("inf")), EINVAL), (dict(position0=(1 << 31) + 1), EINVAL), (dict(position0=-(1 << 31) - 1), EINVAL),
    (dict(q_rows=29), EINVAL), (dict(k_rows=29), EINVAL), (dict(q_out_rows=29), EINVAL), (dict(k_out_rows=1), EINVAL), (dict(k_out_rows=-30), EINVAL),
    (dict(head_dim=80), EUNSUPPORTED), (dict(head_dim=256), EUNSUPPORTED), (dict(seqlen=(1 << 24) + 1), EUNSUPPORTED), (dict(k_out_rows=(1 << 24) + 1), EUNSUPPORTED),
    (dict(batch=16384), EUNSUPPORTED), (dict(batch=16384, heads=2, kv_heads=4), EUNSUPPORTED)], ids=str)
def test_rotary_shapes(lib, kw, status):
    for f in _rope_calls(lib):
        assert _call(f, _rope(**kw), ROPE) == status


@no_device
@pytest.mark.parametrize("dtype,step", [(binding.BF16, 2), (binding.F32, 4)])
def test_rotary_pointers(lib, dtype, step):
    sh = _rope(dtype=dtype)
    for f in _rope_calls(lib):
        assert _call(f, None, ROPE) == EINVAL
        for i in range(5):
            for bad in ([None] if i != 2 else []) + [ROPE[i] + (2 if i == 2 else step // 2)]:       # (keys without a place, or a place without keys)
                ptrs = list(ROPE)
                ptrs[i] = bad
                assert _call(f, sh, ptrs) == EINVAL, (i, bad)
            ptrs = list(ROPE)
            ptrs[i] += 4 if i == 2 else step
            assert _call(f, sh, ptrs) not in (0, EINVAL), i
        # in place, with other rows per slice
        for kw, ptrs in ((dict(q_rows=40), [_at(0), _at(1), None, _at(0), _at(4)]), (dict(k_out_rows=40), [_at(0), _at(1), None, _at(3), _at(1)])):
            assert _call(f, _rope(dtype=dtype, **kw), ptrs) == EINVAL
            kw = {"q_rows": 40, "q_out_rows": 40} if "q_rows" in kw else {"k_rows": 40, "k_out_rows": 40}
            assert _call(f, _rope(dtype=dtype, **kw), ptrs) not in (0, EINVAL)


def test_the_structures_are_laid_out_as_the_header_says(tmp_path):
    """Offset and size of every field, as a C compiler lays the header's structures out."""
    pairs = (("moba_window_shape", binding._CWindowShape), ("moba_rope_shape", binding._CRopeShape))
    lines = []
    for name, c in pairs:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        for field in c._fields_:
            lines.append('printf("%%zu %%zu %%d\\n", offsetof(%s, %s), sizeof(((%s*)0)->%s), _Generic(((%s*)0)->%s, int32_t: 1, int64_t: 2, float: 3, double: 4));'
                         % (name, field[0], name, field[0], name, field[0]))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include <stdint.h>\n#include "moba.h"\nint main(void) {\n%s\nreturn 0; }\n' % "\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    kinds = {ctypes.c_int32: 1, ctypes.c_int64: 2, ctypes.c_float: 3, ctypes.c_double: 4}
    want = []
    for _, c in pairs:
        want.append(str(ctypes.sizeof(c)))
        want += ["%d %d %d" % (getattr(c, n).offset, getattr(c, n).size, kinds[t]) for n, t in c._fields_]
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")[:-1] == want


@no_device
def test_first_key_pointers(lib):
    f = lib.moba_varlen_first_key
    good = (2, ctypes.c_void_p(_at(0)), 5, ctypes.c_void_p(_at(1)), None)
    assert f(*good) not in (0, EINVAL)
    for i, bad in ((0, 0), (0, -1), (1, None), (1, ctypes.c_void_p(_at(0) + 2)), (2, -1), (3, None), (3, ctypes.c_void_p(_at(1) + 1)),
                   (3, ctypes.c_void_p(_at(0)))):
        args = list(good)
        args[i] = bad
        assert f(*args) == EINVAL, (i, bad)


@no_device
def test_rotary_frequencies_beyond_64_bits(lib):
    """An angle that is not finite has no cosine: position times frequency has to be a number, at any position."""
    for kw in (dict(theta=5e-324), dict(theta=1e-308, head_dim=128), dict(scale_factor=1e-307), dict(scale_factor=5e-324),
               dict(theta=1e-200, scale_factor=1e-150), dict(scale_factor=1e-307, orig_len=8192, band_low=1e5, band_high=1e6)):
        for f in _rope_calls(lib):
            assert _call(f, _rope(**kw), ROPE) == EINVAL, kw
    for kw in (dict(theta=1e-200), dict(theta=1e300), dict(scale_factor=1e-200), dict(scale_factor=1e300), dict(theta=5e-324, rot_dim=2),
               dict(scale_factor=1.0, orig_len=1e300)):
        for f in _rope_calls(lib):
            assert _call(f, _rope(**kw), ROPE) not in (0, EINVAL), kw
