"""Gate, norm, scale, residual and next norm: forward and backward against the
fp64 oracle.

Tolerances: fp32 throughout, one rounding at the end.  Sums over a row of H
elements by 64 lanes and over rows by one lane after another err by at most a few
tens of units of 2^-24 of their terms' magnitudes, 4e-6; 1e-5 for fp32 outputs of
a row.  The factors' gradients are sums of N terms of either sign, whose error
grows with the terms' magnitude and not with the sum's: N = 1000 terms sum to
1 / 30 of it, so 1e-4.  A bf16 output adds its own 2^-9: 2^-8.

The gradient through a norm, dp - p mean(dp p), is a difference: in a row of one
element its value is eps / (u^2 + eps) of its terms.  Its error is a matter of the
terms, so its tolerance is stretched by how far it lies below them."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close
from oracle import gated
from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

ROW_TOL, SUM_TOL, BF16_TOL = 1e-5, 1e-4, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
ALL = ("o", "gate", "w_post", "scale", "w_next")


def _inputs(N, H, dtype, stream, parts=ALL, seed=0):
    rng = np.random.default_rng(seed)
    dev = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    v = {"o": dev(N, H).to(dtype), "gate": dev(N, H).to(dtype), "w_post": dev(H), "scale": dev(H),
         "w_next": dev(H)}
    return dev(N, H).to(stream), {k: v[k] for k in parts}, dev(N, H).to(dtype), dev(N, H).to(stream)


def _run(res, v, dy, dres_out, eps=1e-6, backward=True):
    N, H = res.shape
    act = v["o"].dtype if "o" in v else dy.dtype
    nan = lambda like, dtype: torch.full((N, H), float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    out = {}
    if "o" in v:
        out["res_out"] = nan(res, res.dtype)
    if "w_next" in v:
        out["y"] = nan(res, act)
    rstd = torch.full((N, 2), float("nan"), device="cuda")
    am.gated_norm_forward(res, **v, **out, rstd=rstd if backward else None, eps=eps)
    if not backward:
        return out
    grads = {"dres": nan(res, res.dtype)}
    for k, name in (("o", "do"), ("gate", "dgate")):
        if k in v:
            grads[name] = nan(res, act)
    for k in ("w_post", "scale", "w_next"):
        if k in v:
            grads["d" + k] = torch.full((H,), float("nan"), device="cuda")
    ws = torch.full((am.gated_norm_workspace_bytes(N, H),), 0xFF, dtype=torch.uint8, device="cuda")
    dres = grads.pop("dres")
    am.gated_norm_backward(res, rstd, dres, ws, **v, **grads, dy=dy if "w_next" in v else None,
                           dres_out=dres_out, eps=eps)
    return dict(out, dres=dres, **grads)


def _check(res, v, dy, dres_out, eps=1e-6):
    got = _run(res, v, dy, dres_out, eps)
    f = lambda t: None if t is None else t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    n = {k: f(t) for k, t in v.items()}
    R, y, cache = gated.gated_norm_forward(f(res), eps=eps, **n)
    ref = gated.gated_norm_backward(cache, R.shape, dy=f(dy), dres_out=f(dres_out), **n)
    ref.update(res_out=R, y=y)
    # the same without the norm's second term
    flat = dict(cache, p=np.zeros_like(cache["n"])) if "p" in cache else cache
    terms = gated.gated_norm_backward(flat, R.shape, dy=f(dy), dres_out=f(dres_out), **n)
    for name, g in got.items():
        tol = BF16_TOL if g.dtype == BF16 else SUM_TOL if g.dim() == 1 else ROW_TOL
        if name in ("do", "dgate"):
            tol *= max(1.0, np.abs(terms[name]).max() / (np.abs(ref[name]).max() or 1.0))
        assert_close(name, f(g), ref[name], tol)


@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("N,H", [(1, 1), (3, 2), (5, 3), (2, 64), (7, 255), (64, 256), (9, 257), (33, 511),
                                 (64, 768), (10, 1001), (3, 1024), (6, 1025), (5, 1536), (17, 2049),
                                 (3, 4100), (5, 8191), (2, 8192)])
def test_against_oracle(N, H, dtype, stream):
    _check(*_inputs(N, H, dtype, stream, seed=N + H))


@pytest.mark.parametrize("H", [96, 1100])
@pytest.mark.parametrize("parts", [("o", "w_next"), ("o", "gate", "w_next"), ("o", "w_post", "w_next"),
                                   ("o", "scale", "w_next"), ("o", "gate", "scale"), ("o",), ("o", "w_post"),
                                   ("w_next",), ("o", "gate", "w_post", "scale")])
def test_parts_left_out(parts, H):
    res, v, dy, dres_out = _inputs(50, H, BF16, F32, parts, seed=len(parts))
    _check(res, v, dy, dres_out)
    _check(res, v, dy, None)


def test_many_rows():
    """More rows than workgroups take at once."""
    _check(*_inputs(9001, 100, F32, F32))
    _check(*_inputs(5003, 1300, BF16, BF16))


def test_rows_of_zeros_and_large_values():
    res, v, dy, dres_out = _inputs(6, 300, F32, F32, seed=3)
    v["o"][1] = 0
    res[2] = 0
    v["o"][2] = 0
    v["o"][3] *= 1e15  # its squares stay below fp32's largest
    v["gate"][4], v["gate"][5] = -300.0, 300.0
    _check(res, v, dy, dres_out, eps=1e-3)


def test_a_row_that_is_not_finite_stays_alone():
    res, v, dy, dres_out = _inputs(40, 768, BF16, F32, seed=4)
    clean = _run(res, v, dy, dres_out)
    v["o"][11, 5], res[13, 700] = float("nan"), float("inf")
    got = _run(res, v, dy, dres_out)
    keep = torch.tensor([k not in (11, 13) for k in range(40)], device="cuda")
    for name in ("res_out", "y", "dres", "do", "dgate"):
        assert torch.equal(got[name][keep], clean[name][keep]), name


def test_no_rows():
    got = _run(*_inputs(0, 70, BF16, F32))
    for name in ("dw_post", "dscale", "dw_next"):
        assert torch.all(got[name] == 0)


@pytest.mark.parametrize("H,pad", [(64, 1), (77, 3), (768, 8)])
def test_strided_rows_and_in_place(H, pad):
    res, v, dy, dres_out = _inputs(20, H, BF16, F32, seed=5)
    want = _run(res, v, dy, dres_out)
    wide = torch.full((20, 2 * H + pad), 7.0, dtype=BF16, device="cuda")
    o, gate = wide[:, pad:pad + H], wide[:, pad + H:]
    o.copy_(v["o"])
    gate.copy_(v["gate"])
    w = {k: v[k] for k in ("w_post", "scale", "w_next")}
    rstd, y, stream = torch.empty(20, 2, device="cuda"), torch.empty(20, H, dtype=BF16, device="cuda"), res.clone()
    am.gated_norm_forward(stream, o=o, gate=gate, **w, res_out=stream, y=y, rstd=rstd)
    assert torch.equal(stream, want["res_out"]) and torch.equal(y, want["y"])
    dwide = torch.full_like(wide, 7.0)
    do, dgate, d = dwide[:, pad:pad + H], dwide[:, pad + H:], dres_out.clone()
    dw = {"d" + k: torch.empty(H, device="cuda") for k in w}
    ws = torch.empty(am.gated_norm_workspace_bytes(20, H), dtype=torch.uint8, device="cuda")
    am.gated_norm_backward(res, rstd, d, ws, o=o, gate=gate, **w, dy=dy, dres_out=d, do=do, dgate=dgate, **dw)
    assert torch.equal(d, want["dres"]) and torch.equal(do, want["do"]) and torch.equal(dgate, want["dgate"])
    assert all(torch.equal(dw[k], want[k]) for k in dw) and torch.all(dwide[:, :pad] == 7)


def test_rows_past_32_bit_offsets():
    N, H = 2_900_000, 768
    res = torch.empty((N, H), dtype=BF16, device="cuda").normal_()
    assert res.numel() > 1 << 31
    w = torch.rand(H, device="cuda") + 0.5
    out, y = torch.empty_like(res), torch.empty_like(res)
    am.gated_norm_forward(res, o=res, w_post=w, w_next=w, res_out=out, y=y)
    last = res[-5:].clone()
    out2, y2 = torch.empty_like(last), torch.empty_like(last)
    am.gated_norm_forward(last, o=last, w_post=w, w_next=w, res_out=out2, y=y2)
    assert_close("res_out", out[-5:].float().cpu().numpy(), out2.float().cpu().numpy(), BF16_TOL)
    assert_close("y", y[-5:].float().cpu().numpy(), y2.float().cpu().numpy(), BF16_TOL)


def test_same_bits_every_time_and_from_a_graph():
    for N, H in ((5000, 768), (3, 768), (700, 1536)):
        res, v, dy, dres_out = _inputs(N, H, BF16, F32, seed=6)
        first = _run(res, v, dy, dres_out)
        for _ in range(3):
            again = _run(res, v, dy, dres_out)
            assert all(torch.equal(first[k], again[k]) for k in first)
        rstd, ws = torch.empty(N, 2, device="cuda"), torch.empty(am.gated_norm_workspace_bytes(N, H),
                                                                  dtype=torch.uint8, device="cuda")
        out = {k: torch.empty_like(t) for k, t in first.items()}
        fwd = {k: out[k] for k in ("res_out", "y")}
        bwd = {k: out[k] for k in out if k not in fwd and k != "dres"}

        def both():
            am.gated_norm_forward(res, **v, **fwd, rstd=rstd)
            am.gated_norm_backward(res, rstd, out["dres"], ws, **v, **bwd, dy=dy, dres_out=dres_out)

        both()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both()
        for k in range(4):
            res.normal_()
            g.replay()
            torch.cuda.synchronize()
            got = {n: t.clone() for n, t in out.items()}
            both()
            torch.cuda.synchronize()
            assert all(torch.equal(got[n], out[n]) for n in out), k
