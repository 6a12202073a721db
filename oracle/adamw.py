"""AdamW step with 32-bit or 8-bit moments: in exact fp32 operation order (the
definition that the library matches bit for bit) and in fp64.

8-bit moments: blocks of 256 elements share a power-of-two scale that puts the
largest finite magnitude into [128, 256); m and sqrt(v) are codes of 8-bit
floats (4 exponent bits of bias 7, 3 fraction bits) in units of it, rounded down
or up with the probability of what is cut off.
"""

import numpy as np

BLOCK = 256
_F = np.float32


def coefficients(lr, beta1, beta2, eps, step, weight_decay):
    return {"b1": _F(beta1), "c1": _F(1.0 - beta1), "b2": _F(beta2), "c2": _F(1.0 - beta2), "eps": _F(eps),
            "root": _F(1.0 / np.sqrt(1.0 - float(beta2) ** step)),
            "step": _F(lr / (1.0 - float(beta1) ** step)), "keep": _F(1.0 - lr * weight_decay)}


def step_f32(w, g, m, v, k, grad_scale=None):
    """(w, m, v, sqrt(v)): each operation rounded to fp32, in the stated order."""
    w, g, m, v = (np.asarray(t, _F) for t in (w, g, m, v))
    with np.errstate(all="ignore"):
        if grad_scale is not None:
            g = g * _F(grad_scale)
        m = m * k["b1"] + g * k["c1"]
        v = v * k["b2"] + g * g * k["c2"]
        r = np.sqrt(v)
        w = w * k["keep"] - m / (r * k["root"] + k["eps"]) * k["step"]
    return w, m, v, r


def step_f64(w, g, m, v, lr, beta1, beta2, eps, step, weight_decay):
    w, g, m, v = (np.asarray(t, np.float64) for t in (w, g, m, v))
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    up = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w * (1 - lr * weight_decay) - lr * up, m, v


def draws(n, tensor, seed):
    """The 16-bit draws of n elements for m and for sqrt(v)."""
    u = np.uint32
    with np.errstate(over="ignore"):
        x = np.arange(n, dtype=u) * u(0x85EBCA6B) + u((seed + tensor * 0x9E3779B9) & 0xFFFFFFFF)
        x = (x ^ (x >> u(15))) * u(0xD168AAAD)
        x = (x ^ (x >> u(15))) * u(0xAF723597)
        x = x ^ (x >> u(15))
    return (x & u(0xFFFF)).astype(np.int64), (x >> u(16)).astype(np.int64)


def decode(codes, scales):
    """Values (exact in fp32) of uint8 codes."""
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    val = np.where(e == 0, f * 2.0 ** -9, (1.0 + f / 8.0) * 2.0 ** (e - 7.0))
    val = np.where((c & 127) == 127, np.nan, val) * np.where(c & 128, -1.0, 1.0)
    return (val * np.repeat(np.asarray(scales, np.float64), BLOCK)[:c.size]).astype(_F)


def encode(x, bits, least):
    """(codes uint8, scales fp32) of fp32 values, block by block."""
    x = np.asarray(x, _F)
    codes, scales = np.empty(x.size, np.uint8), np.empty(-(-x.size // BLOCK), _F)
    for b in range(scales.size):
        at = slice(b * BLOCK, min(x.size, (b + 1) * BLOCK))
        mag = np.abs(x[at].astype(np.float64))
        finite = mag[np.isfinite(mag)]
        top = float(finite.max()) if finite.size else 0.0
        power = max(np.frexp(top)[1] - 8, -126) if top > 0 else -126
        scales[b] = _F(2.0 ** power)
        with np.errstate(invalid="ignore"):
            y = mag / 2.0 ** power
            unit = np.exp2(np.maximum(np.frexp(y)[1] - 1, -6).astype(np.float64) - 3)
            y = np.where(np.isfinite(y), y, 0.0)
            grid = np.floor(y / unit + bits[at] / 65536.0) * unit  # exact: y / unit < 16, 24 bits
            grid = np.where((y > 0) & (grid < least * 2.0 ** -9), least * 2.0 ** -9, grid)
            ex = np.maximum(np.frexp(np.where(grid > 0, grid, 1.0))[1] - 1, -6)
            normal = grid >= 2.0 ** -6
            c = np.where(normal, ((ex + 7) * 8 + (grid / np.exp2(ex.astype(np.float64)) - 1.0) * 8),
                         grid * 512.0).astype(np.int64)
        c = np.where(np.isfinite(mag), c, 127) | np.where(np.signbit(x[at]), 128, 0)
        codes[at] = c.astype(np.uint8)
    return codes, scales
