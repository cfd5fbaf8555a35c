"""Refusals of the window-attention and rotary entry points: host-side, nothing is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2511_11571_amd as moba
from paper_2511_11571_amd import binding

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
P = 4096                                                      # a pointer that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    return moba.lib()


def _ptr(x):
    return ctypes.c_void_p(x)


def _window(**kw):
    base = dict(batch=2, heads=4, q_len=100, kv_len=300, head_dim=64, window=50, kv_heads=2)
    base.update(kw)
    return moba.WindowShape(**base)


def _sizes(lib, sh):
    a, b = ctypes.c_size_t(7), ctypes.c_size_t(7)
    return lib.moba_window_workspace(ctypes.byref(sh.c()), ctypes.byref(a), ctypes.byref(b)), a.value, b.value


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=3), EINVAL), (dict(kv_heads=-1), EINVAL), (dict(q_len=0), EINVAL),
    (dict(q_len=301), EINVAL), (dict(kv_len=0), EINVAL), (dict(window=-1), EINVAL), (dict(kv_rows=299), EINVAL), (dict(kv_rows=-5), EINVAL),
    (dict(dtype=2), EINVAL), (dict(softmax_scale=float("nan")), EINVAL), (dict(softmax_scale=float("inf")), EINVAL), (dict(head_dim=0), EINVAL),
    (dict(head_dim=96), EUNSUPPORTED), (dict(kv_len=(1 << 24) + 1), EUNSUPPORTED), (dict(kv_rows=(1 << 24) + 1), EUNSUPPORTED),
    (dict(batch=32768, heads=2, kv_heads=0), EUNSUPPORTED)])
def test_window_shapes_that_are_refused(lib, kw, status):
    sh = _window(**kw)
    assert _sizes(lib, sh)[0] == status
    big = ctypes.c_size_t(1 << 40)
    assert lib.moba_window_forward(ctypes.byref(sh.c()), *[_ptr(P)] * 3, None, *[_ptr(P)] * 3, big, None) == status
    assert lib.moba_window_backward(ctypes.byref(sh.c()), *[_ptr(P)] * 6, None, *[_ptr(P)] * 4, big, None) == status


def test_window_pointers_and_workspaces_that_are_refused(lib):
    sh = _window()
    status, fwd, bwd = _sizes(lib, sh)
    assert status == 0 and bwd >= 4 * 2 * 4 * 100
    assert lib.moba_window_workspace(ctypes.byref(sh.c()), None, None) == EINVAL
    assert lib.moba_window_workspace(None, None, None) == EINVAL
    big = ctypes.c_size_t(1 << 40)
    ok = [P] * 8                                              # Q K V first O lse ws | bytes
    for i in (0, 1, 2, 4, 5):
        for bad in (0, P + 8 if i != 5 else P + 2):
            a = [_ptr(bad if j == i else P) for j in range(7)]
            assert lib.moba_window_forward(ctypes.byref(sh.c()), *a, big, None) == EINVAL, i
    assert lib.moba_window_forward(ctypes.byref(sh.c()), *[_ptr(P)] * 3, _ptr(P + 2), *[_ptr(P)] * 3, big, None) == EINVAL
    assert lib.moba_window_forward(ctypes.byref(sh.c()), *[_ptr(P)] * 6, _ptr(P + 8), big, None) == EINVAL
    for i in (0, 1, 2, 3, 4, 5, 7, 8, 9):                     # Q K V O lse dO first dQ dK dV ws
        for bad in (0, P + 8 if i != 4 else P + 2):
            a = [_ptr(bad if j == i else P) for j in range(11)]
            assert lib.moba_window_backward(ctypes.byref(sh.c()), *a, big, None) == EINVAL, i
    a = [_ptr(P)] * 11
    assert lib.moba_window_backward(ctypes.byref(sh.c()), *a, ctypes.c_size_t(bwd - 1), None) == EWORKSPACE
    assert lib.moba_window_backward(ctypes.byref(sh.c()), *a[:10], None, big, None) == EWORKSPACE
    # few queries with a long cache: the keys are shared out, which takes a workspace
    long = _window(batch=1, q_len=1, kv_len=200000, window=0)
    status, fwd, _ = _sizes(lib, long)
    assert status == 0
    if fwd:
        a = [_ptr(P)] * 7
        assert lib.moba_window_forward(ctypes.byref(long.c()), *a, ctypes.c_size_t(fwd - 1), None) == EWORKSPACE
        assert lib.moba_window_forward(ctypes.byref(long.c()), *a[:6], None, big, None) == EWORKSPACE
    assert len(ok) == 8


def test_outputs_that_are_inputs_or_one_another_are_refused(lib):
    sh = _window(batch=1, q_len=1, kv_len=200000, window=0)   # (a call that takes a workspace)
    big = ctypes.c_size_t(1 << 40)
    at = [P * (i + 1) for i in range(11)]
    for outs, n, f in (((4, 5, 6), 7, lib.moba_window_forward), ((7, 8, 9, 10), 11, lib.moba_window_backward)):
        for o in outs:
            for i in range(n):
                if i != o:
                    a = at[:n]
                    a[o] = a[i]
                    assert f(ctypes.byref(sh.c()), *[_ptr(x) for x in a], big, None) == EINVAL, (o, i)
    sh = ctypes.byref(_rope().c())
    for f in (lib.moba_rope, lib.moba_rope_backward):
        for q, k, qo, ko in ((1, 2, 3, 3), (1, 2, 2, 3), (1, 2, 2, 1), (1, 2, 3, 1), (1, 1, 1, 2), (1, 2, 5, 2), (1, 2, 1, 5)):
            assert f(sh, _ptr(q * P), _ptr(k * P), _ptr(5 * P), _ptr(qo * P), _ptr(ko * P), None) == EINVAL


def _rope(**kw):
    base = dict(batch=2, heads=4, seqlen=30, head_dim=64, kv_heads=2)
    base.update(kw)
    return moba.RopeShape(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), EINVAL), (dict(heads=-1), EINVAL), (dict(kv_heads=-1), EINVAL), (dict(seqlen=0), EINVAL), (dict(dtype=3), EINVAL),
    (dict(rot_dim=3), EINVAL), (dict(rot_dim=66), EINVAL), (dict(rot_dim=-2), EINVAL), (dict(interleaved=2), EINVAL), (dict(theta=0.0), EINVAL),
    (dict(theta=float("nan")), EINVAL), (dict(theta=float("inf")), EINVAL), (dict(scale_factor=0.0), EINVAL), (dict(scale_factor=float("nan")), EINVAL),
    (dict(orig_len=-1.0), EINVAL), (dict(orig_len=8192, band_low=4.0, band_high=4.0), EINVAL), (dict(orig_len=8192, band_high=float("inf")), EINVAL),
    (dict(amplitude=float("nan")), EINVAL), (dict(position0=(1 << 31) + 1), EINVAL), (dict(q_rows=29), EINVAL), (dict(k_out_rows=1), EINVAL),
    (dict(head_dim=80), EUNSUPPORTED), (dict(seqlen=(1 << 24) + 1), EUNSUPPORTED), (dict(batch=70000, heads=1), EUNSUPPORTED)])
def test_rope_shapes_that_are_refused(lib, kw, status):
    sh = _rope(**kw).c()
    assert lib.moba_rope(ctypes.byref(sh), _ptr(P), _ptr(P), None, _ptr(P), _ptr(P), None) == status
    assert lib.moba_rope_backward(ctypes.byref(sh), _ptr(P), _ptr(P), None, _ptr(P), _ptr(P), None) == status


def test_rope_pointers_that_are_refused(lib):
    f, sh = lib.moba_rope, ctypes.byref(_rope().c())
    assert f(None, _ptr(P), _ptr(P), None, _ptr(P), _ptr(P), None) == EINVAL
    assert f(sh, None, _ptr(P), None, _ptr(P), _ptr(P), None) == EINVAL
    assert f(sh, _ptr(P), _ptr(P), None, None, _ptr(P), None) == EINVAL
    assert f(sh, _ptr(P), _ptr(P), None, _ptr(P), None, None) == EINVAL            # keys that go nowhere
    assert f(sh, _ptr(P), None, None, _ptr(P), _ptr(P), None) == EINVAL
    assert f(sh, _ptr(P + 1), _ptr(P), None, _ptr(P), _ptr(P), None) == EINVAL
    assert f(sh, _ptr(P), _ptr(P), _ptr(P + 2), _ptr(P), _ptr(P), None) == EINVAL
    apart = ctypes.byref(_rope(q_rows=40).c())               # in place, but with other rows per slice
    assert f(apart, _ptr(P), None, None, _ptr(P), None, None) == EINVAL
    apart = ctypes.byref(_rope(k_out_rows=40).c())
    assert f(apart, _ptr(P), _ptr(2 * P), None, _ptr(P), _ptr(2 * P), None) == EINVAL


def test_first_key_arguments_that_are_refused(lib):
    f = lib.moba_varlen_first_key
    assert f(0, _ptr(P), 5, _ptr(P), None) == EINVAL
    assert f(2, None, 5, _ptr(P), None) == EINVAL
    assert f(2, _ptr(P), -1, _ptr(P), None) == EINVAL
    assert f(2, _ptr(P), 5, None, None) == EINVAL
    assert f(2, _ptr(P), 0, None, None) == 0                  # no rows: nothing to do


def test_the_structures_are_the_headers():
    """Sizes of the two structures as a C compiler lays them out."""
    assert ctypes.sizeof(binding._CWindowShape) == 40
    assert ctypes.sizeof(binding._CRopeShape) == 12 * 4 + 5 * 8 + 8 + 8
