"""The gated delta rule over packed sequences and its gradient, frame by frame in
fp64.

Per head, S [dk][dv]:  q = q / sqrt(q q + eps),  k = k / sqrt(k k + eps),
a_t = exp(-c softplus(lam) sigm(r_t)),  beta_t = sigm(b_t),
S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T,  o_t = S_t^T q_t.
Heads that are neighbours share a pair of q and k.  Frames are packed time-major,
sequences sorted by non-increasing length.
"""

import numpy as np

from oracle.gated import _rows, _sigm, _softplus


def _unit(x, heads, eps):
    """Rows of vectors of unit length, and 1 / their lengths."""
    x = np.asarray(x, np.float64)
    x = x.reshape(len(x), heads, x.shape[1] // heads)
    inv = 1.0 / np.sqrt((x * x).sum(-1, keepdims=True) + eps)
    return x * inv, inv


def gated_delta_forward(q, k, v, r, b, lam, T, B, heads, key_heads, lengths=None, s0=None, c=8.0, eps=1e-6):
    """(o [N][heads dv], sT [B][heads][dk][dv], cache)."""
    each = heads // key_heads
    (q, _), (k, _) = (_unit(x, key_heads, eps) for x in (q, k))
    v = np.asarray(v, np.float64)
    v = v.reshape(len(v), heads, v.shape[1] // heads)
    a = np.exp(-c * _softplus(np.asarray(lam, np.float64)) * _sigm(np.asarray(r, np.float64)))
    beta = _sigm(np.asarray(b, np.float64))
    dk, dv = q.shape[2], v.shape[2]
    S = np.zeros((B, heads, dk, dv)) if s0 is None else np.array(s0, np.float64)
    o, before = np.empty_like(v), []
    for at, nb in _rows(T, B, lengths):
        rows = slice(at, at + nb)
        before.append(S[:nb].copy())
        qt, kt = (np.repeat(x[rows], each, 1) for x in (q, k))
        S[:nb] *= a[rows][:, :, None, None]
        u = beta[rows][:, :, None] * (v[rows] - np.einsum("bhkv,bhk->bhv", S[:nb], kt))
        S[:nb] += kt[..., None] * u[:, :, None, :]
        o[rows] = np.einsum("bhkv,bhk->bhv", S[:nb], qt)
    return o.reshape(len(v), heads * dv), S, {"before": before}


def gated_delta_backward(q, k, v, r, b, lam, T, B, heads, key_heads, d_o, cache, lengths=None, dsT=None, c=8.0,
                         eps=1e-6):
    """(dq, dk, dv, dr, db, dlam, ds0)."""
    each, lam, r = heads // key_heads, np.asarray(lam, np.float64), np.asarray(r, np.float64)
    (qu, qi), (ku, ki) = (_unit(x, key_heads, eps) for x in (q, k))
    N = len(qu)
    v = np.asarray(v, np.float64)
    v = v.reshape(N, heads, v.shape[1] // heads)
    d_o = np.asarray(d_o, np.float64).reshape(v.shape)
    rate, sr, beta = c * _softplus(lam), _sigm(r), _sigm(np.asarray(b, np.float64))
    a = np.exp(-rate * sr)
    dqu, dku, dv = np.zeros_like(qu), np.zeros_like(ku), np.empty_like(v)
    dlog, dbeta = np.empty_like(sr), np.empty_like(sr)  # of log a and of beta
    dS = np.zeros((B, heads, qu.shape[2], v.shape[2])) if dsT is None else np.array(dsT, np.float64)
    shared = lambda x: x.reshape(len(x), key_heads, each, x.shape[2]).sum(2)  # noqa: E731
    for (at, nb), S in reversed(list(zip(_rows(T, B, lengths), cache["before"]))):
        rows = slice(at, at + nb)
        qt, kt = (np.repeat(x[rows], each, 1) for x in (qu, ku))
        at_, bt = a[rows][:, :, None, None], beta[rows][:, :, None]
        D = at_ * S                                   # the state that has decayed
        e = v[rows] - np.einsum("bhkv,bhk->bhv", D, kt)
        after = D + kt[..., None] * (bt * e)[:, :, None, :]
        dqu[rows] += shared(np.einsum("bhkv,bhv->bhk", after, d_o[rows]))
        G = dS[:nb] + qt[..., None] * d_o[rows][:, :, None, :]   # of the new state
        du = np.einsum("bhkv,bhk->bhv", G, kt)
        dbeta[rows] = (du * e).sum(-1)
        dv[rows] = bt * du
        dku[rows] += shared(np.einsum("bhkv,bhv->bhk", G, bt * e) - np.einsum("bhkv,bhv->bhk", D, bt * du))
        dD = G - kt[..., None] * (bt * du)[:, :, None, :]
        dlog[rows] = (dD * D).sum((2, 3))
        dS[:nb] = at_ * dD
    # what the gradients are before their parts along q and k are taken away
    cache["along"] = [float(np.abs(inv * d).max(initial=0.0)) for inv, d in ((qi, dqu), (ki, dku))]
    dq, dk = (inv * (d - u * (u * d).sum(-1, keepdims=True)) for u, inv, d in ((qu, qi, dqu), (ku, ki, dku)))
    return (*(x.reshape(N, x.shape[1] * x.shape[2]) for x in (dq, dk, dv)), dlog * -rate * sr * _sigm(-r),
            dbeta * beta * _sigm(-np.asarray(b, np.float64)), (dlog * -c * sr).sum(0) * _sigm(lam), dS)
