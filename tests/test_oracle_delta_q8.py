"""CPU pins of the oracle's gated delta rule and 8-bit matrices: gradients against
central differences and torch's autograd in fp64, closed forms, a form that joins
chunks, and codes and scales against torch's 8-bit floats."""

import numpy as np
import pytest
import torch

from oracle import delta, q8


def _inputs(T, B, heads, keys, dk, dv, lengths=None, seed=0):
    rng = np.random.default_rng(seed)
    N = T * B if lengths is None else sum(lengths)
    x = [rng.standard_normal((N, n)) for n in (keys * dk, keys * dk, heads * dv, heads, heads)]
    return x + [rng.standard_normal(heads) - 2], rng.standard_normal((B, heads, dk, dv))


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


@pytest.mark.parametrize("lengths,heads,keys", [(None, 2, 2), ([4, 2, 0], 4, 2)])
def test_delta_gradient_is_the_difference_quotient(lengths, heads, keys):
    T, B, dk, dv = 4, 3, 3, 2
    x, s0 = _inputs(T, B, heads, keys, dk, dv, lengths)
    rng = np.random.default_rng(9)
    do, dsT = rng.standard_normal((len(x[0]), heads * dv)), rng.standard_normal(s0.shape)
    sizes = (T, B, heads, keys)

    def total():
        o, sT, _ = delta.gated_delta_forward(*x, *sizes, lengths, s0)
        return float((o * do).sum() + (sT * dsT).sum())

    cache = delta.gated_delta_forward(*x, *sizes, lengths, s0)[2]
    got = delta.gated_delta_backward(*x, *sizes, do, cache, lengths, dsT)
    for g, v in zip(got, (*x, s0)):
        # a central difference of step 1e-6 of values of order 10 in fp64: 1e-8
        np.testing.assert_allclose(g, _difference(total, v), atol=1e-7, rtol=1e-6)


def test_delta_gradient_is_autograds():
    T, B, H, dk, dv = 9, 2, 3, 5, 4
    x, s0 = _inputs(T, B, H, H, dk, dv, seed=3)
    rng = np.random.default_rng(4)
    do, dsT = rng.standard_normal((T * B, H * dv)), rng.standard_normal(s0.shape)
    t = [torch.tensor(v, requires_grad=True) for v in (*x, s0)]
    q, k, v, r, b, lam, S = t
    unit = lambda z: z / torch.sqrt((z * z).sum(-1, keepdim=True) + 1e-6)  # noqa: E731
    q, k, v = unit(q.view(T, B, H, dk)), unit(k.view(T, B, H, dk)), v.view(T, B, H, dv)
    a = torch.exp(-8 * torch.nn.functional.softplus(lam) * torch.sigmoid(r.view(T, B, H)))
    beta, out = torch.sigmoid(b.view(T, B, H)), []
    for n in range(T):
        S = S * a[n][..., None, None]
        S = S + torch.einsum("bhk,bhv->bhkv", k[n], beta[n][..., None] * (v[n] - torch.einsum("bhkv,bhk->bhv", S, k[n])))
        out.append(torch.einsum("bhkv,bhk->bhv", S, q[n]))
    o = torch.stack(out).reshape(T * B, -1)
    want = torch.autograd.grad((o * torch.tensor(do)).sum() + (S * torch.tensor(dsT)).sum(), t)
    oo, sT, cache = delta.gated_delta_forward(*x, T, B, H, H, None, s0)
    np.testing.assert_allclose(oo, o.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(sT, S.detach().numpy(), rtol=1e-12, atol=1e-13)
    for g, w in zip(delta.gated_delta_backward(*x, T, B, H, H, do, cache, None, dsT), want):
        np.testing.assert_allclose(g, w.numpy().reshape(g.shape), rtol=1e-10, atol=1e-11)


def test_delta_closed_forms():
    # orthonormal keys, gates open and nothing forgotten: what was written is read back
    T = dk = 6
    k, v = np.eye(T), np.random.default_rng(1).standard_normal((T, 3))
    far = np.full((T, 1), 800.0)
    o, S, _ = delta.gated_delta_forward(k, k, v, -far, far, np.zeros(1), T, 1, 1, 1, eps=1e-30)
    np.testing.assert_allclose(o, v, atol=1e-14)
    np.testing.assert_allclose(S[0, 0], v, atol=1e-14)
    # the same key again replaces what it held
    k = np.tile([[1.0, 2.0]], (T, 1))
    o, S, _ = delta.gated_delta_forward(k, k, v, -far, far, np.zeros(1), T, 1, 1, 1, eps=1e-30)
    np.testing.assert_allclose(o, v, atol=1e-14)
    # a shut gate writes nothing, and the state decays by a
    o, S, _ = delta.gated_delta_forward(k, k, v, np.zeros((T, 1)), -far, np.zeros(1), T, 1, 1, 1, s0=np.ones((1, 1, 2, 3)))
    np.testing.assert_allclose(S, np.exp(-8 * np.log(2.0) / 2 * T), rtol=1e-13)


def test_delta_carried_state():
    T, B, H = 12, 2, 2
    x, s0 = _inputs(T, B, H, 1, 4, 3, seed=5)
    o, sT, _ = delta.gated_delta_forward(*x, T, B, H, 1, None, s0)
    cut = [v[:5 * B] for v in x[:5]], [v[5 * B:] for v in x[:5]]
    o1, s1, _ = delta.gated_delta_forward(*cut[0], x[5], 5, B, H, 1, None, s0)
    o2, s2, _ = delta.gated_delta_forward(*cut[1], x[5], T - 5, B, H, 1, None, s1)
    assert np.array_equal(np.concatenate([o1, o2]), o) and np.array_equal(s2, sT)


def test_delta_is_the_chunked_form():
    """One chunk by its triangular system: U = (I + L)^-1 diag(beta)(V - diag(g) K S)."""
    T, dk, dv = 17, 5, 3
    x, s0 = _inputs(T, 1, 1, 1, dk, dv, seed=6)
    q, k, v, r, b, lam = x
    o, sT, _ = delta.gated_delta_forward(*x, T, 1, 1, 1, None, s0)
    unit = lambda z: z / np.sqrt((z * z).sum(-1, keepdims=True) + 1e-6)  # noqa: E731
    q, k, S = unit(q), unit(k), s0[0, 0]
    c = np.cumsum(-8 * np.logaddexp(0, lam[0]) / (1 + np.exp(-r[:, 0])))
    beta, g = 1 / (1 + np.exp(-b)), np.exp(c)[:, None]
    M = np.tril(np.exp(c[:, None] - c[None, :]))
    U = np.linalg.solve(np.eye(T) + np.tril(beta * M * (k @ k.T), -1), beta * (v - g * (k @ S)))
    np.testing.assert_allclose(g * (q @ S) + (M * (q @ k.T)) @ U, o, atol=1e-12)
    np.testing.assert_allclose(g[-1] * S + (k * np.exp(c[-1] - c)[:, None]).T @ U, sT[0, 0], atol=1e-12)


def test_q8_values_are_torchs():
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code.copy()).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(q8.value(code), want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = (rng.standard_normal(100000) * np.exp2(rng.integers(-16, 7, 100000))).astype(np.float32)
    x = np.concatenate([x[np.abs(x) < 256], np.float32([0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17, 19, 21, 255.9])])
    want = torch.from_numpy(x.copy()).to(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(q8.nearest(x), want)


@pytest.mark.parametrize("tiles", [False, True])
def test_q8_scales(tiles):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 300)) * np.exp(rng.standard_normal((200, 1)) * 3)
    x[:3], x[5, :128], x[6, 3] = 0, 0, np.inf
    v, e = q8.quantise(x, tiles)
    assert e.shape == ((2, 3) if tiles else (200, 3))
    scale = q8.spread(e, x.shape, tiles)
    fine = np.isfinite(x)
    assert np.abs(x[fine] / scale[fine]).max() < 256 and np.isnan(v[6, 3])
    # half a step of a normal code is 2^-4 of it, of a subnormal one 2^-10
    assert np.all(np.abs(v - x / scale)[fine] <= np.maximum(np.abs(x / scale)[fine] * 2.0 ** -4, 2.0 ** -10))
    if not tiles:
        top = np.abs(np.where(fine, x, 0))[:, :128].max(1) / scale[:, 0]
        assert np.all((top >= 128) | (e[:, 0] == 1))
