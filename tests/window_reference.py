"""Attention to the last W keys, its gradients and rotary positions in 64 bits, from the formulas, with bounds on
how far a computation in the I/O type may be off.

A rounding to the I/O type is off by at most half a step, h |x| with h = finfo.eps / 2; sums and products in
between are in 32 bits, u = 2^-24.  With S = scale q.k and E = (d + 8) u (scale |q|.|k|) its error:
  P = exp(S - lse) is off by a factor 1 + e_p, e_p = max E of the row + n u + 4 u (1 + |S| + |lse|) + h (P enters its
      products in the I/O type; n keys in the sums)
  O    e_p sum(P |v|) + h |O|,  and the sums' own error n u sum(P |v|)
  D    |dO| . (error of O)  (D is taken from the stored O) + d u |dO| . |O|
  dS   |dS| (e_p + h) + P (d u |dO|.|v| + error of D)
  gradients: products of these errors with the magnitudes of the other operand, and their own rounding.
"""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def seen(q, N, W, first, batch):
    """[batch, q, N]: does the row attend the key"""
    t = np.arange(N - q, N)[:, None]
    u = np.arange(N)[None, :]
    m = (u <= t) & (u > t - (W or N))
    m = np.broadcast_to(m, (batch, q, N))
    if first is not None:
        m = m & (u[None] >= np.asarray(first)[:, :, None])
    return m


def window(Q, K, V, W, first, scale=None, dO=None):
    """Tensors as handed to the library (K, V cut to N rows), results {name: (value, bound)} as float64 arrays."""
    dt = Q.dtype
    h = half_step(dt) if dt != torch.float32 else 0.0        # an fp32 result's rounding is among the u
    hs = half_step(dt)
    q_, k_, v_ = (x.detach().cpu().double().numpy() for x in (Q, K, V))
    b, H, q, d = q_.shape
    G, N = H // k_.shape[1], k_.shape[2]
    scale = scale if scale else 1.0 / np.sqrt(d)
    k_, v_ = np.repeat(k_, G, 1), np.repeat(v_, G, 1)
    on = np.broadcast_to(seen(q, N, W, None if first is None else first.cpu().numpy(), b)[:, None], (b, H, q, N))
    kz, vz = np.where(np.isfinite(k_), k_, 0.0), np.where(np.isfinite(v_), v_, 0.0)
    qz = np.where(np.isfinite(q_), q_, 0.0)
    S = scale * (qz @ kz.swapaxes(-1, -2))
    aS = scale * (np.abs(qz) @ np.abs(kz).swapaxes(-1, -2))
    any_on = on.any(-1)
    Sm = np.where(on, S, -np.inf)
    top = np.where(any_on, Sm.max(-1), 0.0)
    e = np.where(on, np.exp(Sm - top[..., None]), 0.0)
    l = e.sum(-1)
    P = e / np.where(any_on, l, 1.0)[..., None]
    with np.errstate(divide="ignore"):
        lse = np.where(any_on, top + np.log(l), -np.inf)
    n = on.sum(-1)
    E = np.where(on, (d + 8) * U * aS, 0.0).max(-1) if N else 0.0
    big = np.where(on, np.abs(S), 0.0).max(-1) + np.where(any_on, np.abs(np.where(any_on, lse, 0.0)), 0.0)
    ep = 2 * (E + 4 * U * (1 + big)) + n * U + h
    O, aO = P @ vz, P @ np.abs(vz)
    eO = (ep + n * U)[..., None] * aO + hs * np.abs(O)
    out = {"O": (O, eO + 1e-30), "lse": (lse, np.where(any_on, E + (n + 8) * U + 8 * U * big, 0.0))}
    if dO is None:
        return out
    g = dO.detach().cpu().double().numpy()
    g = np.where(np.isfinite(g), g, 0.0) * any_on[..., None]
    dP, adP = g @ vz.swapaxes(-1, -2), np.abs(g) @ np.abs(vz).swapaxes(-1, -2)
    D = (g * O).sum(-1)
    eD = (np.abs(g) * eO).sum(-1) + (d + 8) * U * (np.abs(g) * np.abs(O)).sum(-1)
    dS = P * (dP - D[..., None])
    edS = np.abs(dS) * (ep + h)[..., None] + P * ((d + 8) * U * adP + eD[..., None] + 4 * U * np.abs(D)[..., None])
    fold = lambda x: x.reshape(b, H // G, G, N, d).sum(2)  # noqa: E731
    dQ, edQ = scale * dS @ kz, scale * (edS + n[..., None] * U * np.abs(dS)) @ np.abs(kz)
    T = lambda x: x.swapaxes(-1, -2)  # noqa: E731
    m = on.sum(-2) * G
    dK = fold(scale * T(dS) @ qz)
    edK = fold(scale * T(edS) @ np.abs(qz) + (m[..., None] * U) * (scale * T(np.abs(dS)) @ np.abs(qz)))
    dV = fold(T(P) @ g)
    edV = fold(T(P * ep[..., None]) @ np.abs(g) + (m[..., None] * U) * (T(P) @ np.abs(g)))
    for name, x, ex in (("dQ", dQ, edQ), ("dK", dK, edK), ("dV", dV, edV)):
        out[name] = (x, ex + hs * np.abs(x) + 1e-30)
    return out


def close(got, want, name, rows=None):
    value, bound = want
    a = got.detach().cpu().double().numpy()
    if rows is not None:
        a = a[:, :, :rows]
    assert a.shape == value.shape, name
    same = a == value                                        # (infinities)
    off = np.where(same, 0.0, np.abs(a - np.where(same, 0.0, value)))
    worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off - bound)), off.shape)
    assert np.all(off <= bound), f"{name}{worst}: {a[worst]} is not {value[worst]}, off {off[worst]:.3g}, bound {bound[worst]:.3g}"


def rope(x, positions, rot, interleaved, freq, amplitude, back=False):
    """x [b,h,N,d] tensor, positions [b,N] float64, freq in radians -> value, magnitude |x| + |y| of every channel's pair"""
    a = x.detach().cpu().double().numpy()
    ang = positions[:, None, :, None] * np.asarray(freq)
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang) * (-1 if back else 1)
    out, mag = a.copy(), np.abs(a)
    i = np.arange(rot // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    out[..., p] = a[..., p] * c - a[..., q] * s
    out[..., q] = a[..., q] * c + a[..., p] * s
    mag[..., p] = mag[..., q] = np.abs(amplitude) * (np.abs(a[..., p]) + np.abs(a[..., q]))
    return out, mag


def rope_frequencies(sh):
    f = []
    rot = sh.rot_dim or sh.head_dim
    for i in range(rot // 2):
        g = sh.theta ** (-2.0 * i / rot)
        keep = 0.0
        if sh.orig_len > 0:
            keep = min(1.0, max(0.0, (sh.orig_len * g / (2 * np.pi) - sh.band_low) / (sh.band_high - sh.band_low)))
        f.append(g * (keep + (1 - keep) / sh.scale_factor))
    return f
