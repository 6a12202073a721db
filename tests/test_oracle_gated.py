"""CPU pins of the oracle's gated recurrence, norms and AdamW step: gradients
against central differences and torch's autograd in fp64, closed forms, and the
8-bit codes against torch's float8_e4m3fn."""

import numpy as np
import pytest
import torch

from oracle import adamw, gated


def _difference(f, v, h=1e-6):
    g = np.empty_like(v)
    for k in np.ndindex(*v.shape):
        keep = v[k]
        v[k] = keep + h
        hi = f()
        v[k] = keep - h
        lo = f()
        v[k] = keep
        g[k] = (hi - lo) / (2 * h)
    return g


@pytest.mark.parametrize("lengths", [None, [5, 3, 3, 0]])
def test_recurrence_gradient_is_the_difference_quotient(lengths):
    rng = np.random.default_rng(1)
    T, B, H = 5, 4, 3
    N = T * B if lengths is None else sum(lengths)
    x, r, i, dh = (rng.standard_normal((N, H)) for _ in range(4))
    lam, h0, dhT = rng.standard_normal(H) - 2, rng.standard_normal((B, H)), rng.standard_normal((B, H))

    def total():
        h, hT, _ = gated.gated_recurrence_forward(x, r, i, lam, T, B, lengths, h0)
        return float((h * dh).sum() + (hT * dhT).sum())

    _, _, cache = gated.gated_recurrence_forward(x, r, i, lam, T, B, lengths, h0)
    got = gated.gated_recurrence_backward(x, r, i, lam, T, B, dh, cache, lengths, dhT)
    for g, v in zip(got, (x, r, i, lam, h0)):
        # a central difference of step 1e-6 of values of order 10 in fp64: 1e-8
        np.testing.assert_allclose(g, _difference(total, v), atol=1e-7, rtol=1e-6)


def test_recurrence_closed_forms():
    # a constant gate and input: the geometric series
    T, c = 40, 8.0
    lam, r, i, x = np.array([-1.0]), np.full((T, 1), 0.3), np.full((T, 1), -0.2), np.full((T, 1), 1.5)
    h, hT, _ = gated.gated_recurrence_forward(x, r, i, lam, T, 1, c=c)
    a = np.exp(-c * np.log1p(np.exp(-1.0)) / (1 + np.exp(-0.3)))
    u = np.sqrt(1 - a * a) * 1.5 / (1 + np.exp(0.2))
    np.testing.assert_allclose(h[:, 0], u * (1 - a ** np.arange(1, T + 1)) / (1 - a), rtol=1e-12)
    # a shut gate keeps the state, an open one at a high rate forgets it
    h, _, _ = gated.gated_recurrence_forward(x, np.full((T, 1), -np.inf), i, lam, T, 1, h0=np.array([[2.0]]))
    assert np.all(h == 2.0)


def test_norm_gradient_is_autograds():
    rng = np.random.default_rng(2)
    N, H, eps = 6, 9, 1e-3
    v = {k: rng.standard_normal((N, H)) for k in ("o", "gate", "res")}
    v.update({k: rng.standard_normal(H) for k in ("w_post", "scale", "w_next")})
    dy, dres_out = rng.standard_normal((N, H)), rng.standard_normal((N, H))
    t = {k: torch.tensor(a, requires_grad=True) for k, a in v.items()}
    u = t["o"] * torch.nn.functional.silu(t["gate"])
    R = t["res"] + t["scale"] * t["w_post"] * u * torch.rsqrt(u.pow(2).mean(1, keepdim=True) + eps)
    y = t["w_next"] * R * torch.rsqrt(R.pow(2).mean(1, keepdim=True) + eps)
    ((y * torch.tensor(dy)).sum() + (R * torch.tensor(dres_out)).sum()).backward()
    R2, y2, cache = gated.gated_norm_forward(**v, eps=eps)
    np.testing.assert_allclose(R2, R.detach().numpy(), rtol=1e-12)
    np.testing.assert_allclose(y2, y.detach().numpy(), rtol=1e-12)
    got = gated.gated_norm_backward(cache, (N, H), v["o"], v["gate"], v["w_post"], v["scale"], v["w_next"],
                                    dy, dres_out)
    for k, name in (("o", "do"), ("gate", "dgate"), ("res", "dres"), ("w_post", "dw_post"),
                    ("scale", "dscale"), ("w_next", "dw_next")):
        np.testing.assert_allclose(got[name], t[k].grad.numpy(), rtol=1e-10, atol=1e-12)


def test_adamw_step_is_torchs():
    rng = np.random.default_rng(3)
    n, opt = 50, dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)
    w = rng.standard_normal(n)
    t = torch.tensor(w, requires_grad=True)
    ref = torch.optim.AdamW([t], lr=opt["lr"], betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    w64, m64, v64 = w, np.zeros(n), np.zeros(n)
    w32, m32, v32 = w.astype(np.float32), np.zeros(n, np.float32), np.zeros(n, np.float32)
    for step in range(1, 6):
        g = rng.standard_normal(n)
        t.grad = torch.tensor(g)
        ref.step()
        w64, m64, v64 = adamw.step_f64(w64, g, m64, v64, step=step, **opt)
        w32, m32, v32, _ = adamw.step_f32(w32, g.astype(np.float32), m32, v32,
                                          adamw.coefficients(step=step, **opt))
        np.testing.assert_allclose(w64, t.detach().numpy(), rtol=1e-12, atol=1e-14)
        np.testing.assert_allclose(w32, w64, rtol=2e-6, atol=1e-6)


def test_codes_are_the_8_bit_floats():
    every = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(every.copy()).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(adamw.decode(every, [1.0]), ref)


def test_codes_round_trip_and_bracket():
    rng = np.random.default_rng(4)
    x = (rng.standard_normal(1000) * np.exp(rng.uniform(-14, 2, 1000))).astype(np.float32)
    lo, s = adamw.encode(x, np.zeros(1000, np.int64), 0)
    hi, _ = adamw.encode(x, np.full(1000, 65535), 0)
    low, high = np.abs(adamw.decode(lo, s)), np.abs(adamw.decode(hi, s))
    assert np.all(low <= np.abs(x)) and np.all(high >= np.abs(x) * (1 - 2.0 ** -15))
    # neighbours on the grid, and values on it stay there whatever the draw
    unit = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(low / np.repeat(s, 256)[:1000], 2.0 ** -6))) - 3), 2.0 ** -9)
    assert np.all(high - low <= unit * np.repeat(s, 256)[:1000] * (1 + 1e-6))
    kept, s2 = adamw.encode(adamw.decode(lo, s), np.full(1000, 65535), 0)
    np.testing.assert_array_equal(adamw.decode(kept, s2), adamw.decode(lo, s))


def test_rounding_is_unbiased():
    n = 1 << 18
    for_m, for_v = adamw.draws(n, 3, 77)
    x = np.full(n, 1.2345, np.float32)
    x[::256] = 200.0  # the blocks' largest: the scale is 1
    for bits in (for_m, for_v):
        c, s = adamw.encode(x, bits, 0)
        y = adamw.decode(c, s).astype(np.float64)
        assert np.all(s == 1.0)
        # steps of 1/8 between 1.125 and 1.25: deviation 0.042 each, 5 sigma of the mean
        assert abs(np.delete(y, np.s_[::256]).mean() - 1.2345) < 5 * 0.063 / np.sqrt(n)


def test_a_nonzero_root_keeps_a_code():
    x = np.zeros(256, np.float32)
    x[0], x[1], x[2] = 1.0, 1e-7, 1e-30
    c, _ = adamw.encode(x, np.zeros(256, np.int64), 1)
    assert c[1] == 1 and c[2] == 1 and c[3] == 0
