"""Gated linear recurrence over packed sequences, the norms around it, and their
gradients, in fp64.

Recurrence, per channel: L_t = c softplus(lam) sigm(r_t), a_t = exp(-L_t),
h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigm(i_t) x_t.  Frames are packed
time-major, sequences sorted by non-increasing length.

Norms, per row: u = o * gate * sigm(gate), p = u / rms(u), R = res + scale *
w_post * p, y = w_next * R / rms(R), rms(z) = sqrt(mean(z^2) + eps).
"""

import numpy as np


def _sigm(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def _softplus(z):
    return np.logaddexp(0.0, z)


def _rows(T, B, lengths):
    """(first row, active sequences) of every frame."""
    lens = [T] * B if lengths is None else [int(v) for v in lengths]
    out, at = [], 0
    for t in range(max(lens, default=0)):
        nb = sum(n > t for n in lens)
        out.append((at, nb))
        at += nb
    return out


def _gates(r, lam, c):
    rate = c * _softplus(np.asarray(lam, np.float64))
    sr = _sigm(r)
    L = rate * sr
    return sr, L, np.exp(-L), np.sqrt(-np.expm1(-2.0 * L))


def gated_recurrence_forward(x, r, i, lam, T, B, lengths=None, h0=None, c=8.0):
    """(h [N][H], hT [B][H], cache)."""
    x, r, i = (np.asarray(v, np.float64) for v in (x, r, i))
    H = x.shape[1]
    _, _, a, q = _gates(r, lam, c)
    u = q * _sigm(i) * x
    state = np.zeros((B, H)) if h0 is None else np.array(h0, np.float64)
    h, before = np.empty_like(x), np.empty_like(x)
    for at, nb in _rows(T, B, lengths):
        before[at:at + nb] = state[:nb]
        state[:nb] = a[at:at + nb] * state[:nb] + u[at:at + nb]
        h[at:at + nb] = state[:nb]
    return h, state, {"before": before}


def gated_recurrence_backward(x, r, i, lam, T, B, dh, cache, lengths=None, dhT=None, c=8.0):
    """(dx, dr, di, dlam, dh0)."""
    x, r, i, dh = (np.asarray(v, np.float64) for v in (x, r, i, dh))
    lam = np.asarray(lam, np.float64)
    sr, L, a, q = _gates(r, lam, c)
    si = _sigm(i)
    carry = np.zeros((B, x.shape[1])) if dhT is None else np.array(dhT, np.float64)
    d = np.empty_like(x)
    for at, nb in reversed(_rows(T, B, lengths)):
        d[at:at + nb] = dh[at:at + nb] + carry[:nb]
        carry[:nb] = a[at:at + nb] * d[at:at + nb]
    v = si * x
    # dL/d(log a) times log a; L / q -> 0 where the gate is shut
    Lq = np.divide(L, q, out=np.zeros_like(L), where=q > 0)
    e = d * (v * a * a * Lq - L * a * cache["before"])
    dv = d * q
    ratio = np.where(lam < -30, 1.0, _sigm(lam) / np.maximum(_softplus(lam), 1e-300))
    return dv * si, e * (1.0 - sr), dv * x * si * (1.0 - si), e.sum(0) * ratio, carry


def gated_norm_forward(res, o=None, gate=None, w_post=None, scale=None, w_next=None, eps=1e-6):
    """(res_out, y, cache); y is None without w_next."""
    R = np.array(res, np.float64)
    f = lambda w: 1.0 if w is None else np.asarray(w, np.float64)  # noqa: E731
    cache = {}
    if o is not None:
        u = np.asarray(o, np.float64)
        if gate is not None:
            gate = np.asarray(gate, np.float64)
            u = u * gate * _sigm(gate)
        ru = 1.0 if w_post is None else 1.0 / np.sqrt((u * u).mean(1, keepdims=True) + eps)
        cache.update(p=u * ru, ru=ru)
        R = R + f(scale) * f(w_post) * u * ru
    rn = 1.0 if w_next is None else 1.0 / np.sqrt((R * R).mean(1, keepdims=True) + eps)
    cache.update(n=R * rn, rn=rn)
    return R, None if w_next is None else R * rn * f(w_next), cache


def gated_norm_backward(cache, res_shape, o=None, gate=None, w_post=None, scale=None, w_next=None, dy=None,
                        dres_out=None):
    """dict of do, dgate, dres, dw_post, dscale, dw_next (those that exist)."""
    f = lambda w: 1.0 if w is None else np.asarray(w, np.float64)  # noqa: E731
    d = np.zeros(res_shape) if dres_out is None else np.array(dres_out, np.float64)
    out = {}
    if w_next is not None:
        dy = np.asarray(dy, np.float64)
        n, dn = cache["n"], dy * f(w_next)
        d = d + cache["rn"] * (dn - n * (dn * n).mean(1, keepdims=True))
        out["dw_next"] = (dy * n).sum(0)
    out["dres"] = d
    if o is not None:
        p, dp = cache["p"], d * f(scale) * f(w_post)
        if w_post is not None:
            out["dw_post"] = (d * p).sum(0) * f(scale)
            du = cache["ru"] * (dp - p * (dp * p).mean(1, keepdims=True))
        else:
            du = dp
        if scale is not None:
            out["dscale"] = (d * p).sum(0) * f(w_post)
        if gate is None:
            out["do"] = du
        else:
            g = np.asarray(gate, np.float64)
            s = _sigm(g)
            out["do"] = du * g * s
            out["dgate"] = du * np.asarray(o, np.float64) * s * (1.0 + g * (1.0 - s))
    return out
