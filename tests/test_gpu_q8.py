"""Matrices in 8 bits: quantising bit for bit, products and the norm against the fp64
oracle.

Products of two codes are exact.  The matrix cores add 128 of them keeping 12 bits below
the largest at least (a probe with magnitudes over the codes' whole range found 2^-13 of
the sum of magnitudes), and the sums of the blocks in 32 bits; one rounding to bf16 is
half a step, 2^-8 of the value: |error| <= 2^-8 |out| + 2^-12 sum |a| |b|."""

import numpy as np
import pytest
import torch

from oracle import gated, q8
from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
SIZES = [(1, 1), (1, 16), (3, 17), (127, 128), (128, 129), (130, 15), (64, 2304), (257, 500), (300, 127), (1000, 8)]


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _matrix(R, C, dtype, seed=0, spread=3.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, C)) * np.exp(rng.standard_normal((R, 1)) * spread)
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)


def _room(rows, cols, tiles=False):
    """q8_empty with every byte 0xFF, so that what is written shows."""
    codes, scales = am.q8_empty(rows, cols, tiles)
    codes.untyped_storage().fill_(0xFF)
    scales.untyped_storage().fill_(0xFF)
    return codes, scales


def _whole(codes):
    """All bytes of the rows, those behind their ends too."""
    rows, stride = codes.shape[0], codes.stride(0)
    return torch.as_strided(codes.view(torch.uint8), (rows, stride), (stride, 1)).cpu().numpy()


def _check(codes, scales, x, tiles):
    """Codes and scales of x [rows][cols] in fp64, bit for bit."""
    value, e = q8.quantise(x, tiles)
    R, C = x.shape
    raw = _whole(codes)
    assert np.array_equal(q8.value(raw[:, :C]), value, equal_nan=True)
    assert np.all(raw[:, C:] == 0)
    used = scales.view(torch.uint8).cpu().numpy()
    assert np.array_equal(used[:, :e.shape[1]], e)
    assert np.all(used[:, e.shape[1]:] == 0xFF)  # bytes that serve nothing are left


@BOTH
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantise(R, C, tiles, dtype):
    x = _matrix(R, C, dtype, seed=R + C)
    at, back = _room(R, C, tiles), _room(C, R, tiles)
    am.q8_quantise(x, *at, *back, tiles=tiles)
    _check(*at, _f64(x), tiles)
    _check(*back, _f64(x).T, tiles)
    # each of the two alone
    one, other = _room(R, C, tiles), _room(C, R, tiles)
    am.q8_quantise(x, *one, tiles=tiles)
    am.q8_quantise(x, codes_t=other[0], scales_t=other[1], tiles=tiles)
    assert np.array_equal(_whole(one[0]), _whole(at[0])) and np.array_equal(_whole(other[0]), _whole(back[0]))


@BOTH
@pytest.mark.parametrize("pad", [1, 4, 8])
def test_quantise_columns_of_a_wider_matrix(pad, dtype):
    x = _matrix(140, 200 + 2 * pad, dtype, seed=pad)[:, pad:pad + 200]
    at, back = _room(140, 200), _room(200, 140)
    am.q8_quantise(x, *at, *back)
    _check(*at, _f64(x), False)
    _check(*back, _f64(x).T, False)


def test_quantise_special_values():
    x = _matrix(130, 300, torch.float32, seed=1)
    x[0], x[1, :128] = 0.0, 0.0
    x[2, 5], x[3, 7], x[4, 9] = float("inf"), float("-inf"), float("nan")
    x[5, :] = float("nan")
    x[6] = 1e-42           # subnormal
    x[7, :128] = 3.3e38
    x[8, :4] = torch.tensor([128.0, 17 / 16, 19 / 16, -21 / 16])  # ties of codes in units of 1
    x[8, 4:128] = 0.0
    x[9, :128] = -0.0
    at, back = _room(130, 300), _room(300, 130)
    am.q8_quantise(x, *at, *back)
    _check(*at, _f64(x), False)
    _check(*back, _f64(x).T, False)


def _operands(M, N, K, tiles, seed=0):
    a, b = am.q8_empty(M, K), am.q8_empty(N, K, tiles)
    am.q8_quantise(_matrix(M, K, torch.float32, seed, 0.5), *a)
    am.q8_quantise(_matrix(N, K, torch.float32, seed + 1, 0.5), *b, tiles=tiles)
    value = lambda m, t: (q8.value(m[0].view(torch.uint8).cpu().numpy()) *  # noqa: E731
                          q8.spread(m[1].view(torch.uint8).cpu().numpy()[:, :-(-K // 128)], m[0].shape, t))
    return a, b, value(a, False), value(b, tiles)


def _close(out, a, b, extra=0.0):
    ref, size = a @ b.T + extra, np.abs(a) @ np.abs(b).T + np.abs(extra)
    err = np.abs(_f64(out) - ref)
    assert np.all(err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -12 * size), float((err / (np.abs(ref) + 1e-30)).max())


def _product(a, b, out, **kw):
    need = am.q8_matmul_workspace_bytes(a[0].shape[0], b[0].shape[0], a[0].shape[1])
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    am.q8_matmul(*a, *b, out, ws=ws, **kw)


# (the last ones: several sums of one output, tiles of 128 and of 256 rows)
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 16), (64, 64, 128), (65, 63, 127), (16, 200, 129), (64, 2304, 768),
                                   (130, 257, 640), (129, 128, 511), (33, 70, 1100), (300, 500, 5000), (200, 100, 4097),
                                   (1500, 1400, 300), (1030, 1100, 8200), (8200, 8200, 136)])
def test_product(M, N, K, tiles):
    a, b, va, vb = _operands(M, N, K, tiles, seed=M + N + K)
    out = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    _product(a, b, out, tiles=tiles)
    if M * N > 1 << 22:  # every row and column of tiles, without the whole product in fp64
        rows, cols = np.arange(0, M, 37), np.arange(0, N, 41)
        _close(out[rows][:, cols], va[rows], vb[cols])
        assert torch.isfinite(out).all()
    else:
        _close(out, va, vb)


@pytest.mark.parametrize("M,N,K", [(70, 130, 300), (64, 64, 4500), (300, 256, 64)])
def test_product_with_bias_and_accumulation(M, N, K):
    a, b, va, vb = _operands(M, N, K, True, seed=K)
    bias = torch.randn(N, device="cuda")
    before = torch.randn((M, N), device="cuda").to(torch.bfloat16)
    out = before.clone()
    _product(a, b, out, tiles=True, bias=bias, accumulate=True)
    _close(out, va, vb, _f64(before) + _f64(bias))


@pytest.mark.parametrize("pad", [1, 3, 8])
def test_product_into_columns(pad):
    M, N, K = 77, 90, 200
    a, b, va, vb = _operands(M, N, K, False, seed=pad)
    wide = torch.full((M, N + 2 * pad), 7.0, dtype=torch.bfloat16, device="cuda")
    _product(a, b, wide[:, pad:pad + N])
    _close(wide[:, pad:pad + N], va, vb)
    assert torch.all(wide[:, :pad] == 7) and torch.all(wide[:, pad + N:] == 7)


def test_product_without_a_sum():
    a, b = am.q8_empty(5, 0), am.q8_empty(7, 0)
    out, bias = torch.full((5, 7), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.arange(7.0, device="cuda")
    _product(a, b, out, bias=bias)
    assert torch.equal(out, bias.to(torch.bfloat16).expand(5, 7))
    _product(*[am.q8_empty(0, 40), am.q8_empty(7, 40)], torch.empty((0, 7), dtype=torch.bfloat16, device="cuda"))


def test_a_nan_stays_in_its_row_and_rooms_of_two_calls():
    M, N, K = 100, 90, 4500
    a, b, _, _ = _operands(M, N, K, False, seed=3)
    clean, out = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _product(a, b, clean)
    a[0].view(torch.uint8)[13, 4499] = 0x7F
    _product(a, b, out)
    _product(a, b, torch.empty_like(out))
    rows = torch.isnan(out).any(1).nonzero().flatten().tolist()
    assert rows == [13] and torch.isnan(out[13]).all()
    out[13] = clean[13]
    assert torch.equal(out, clean)


def test_gradients_of_a_projection():
    """y = x w^T in 8 bits, dx = dy w and dw = dy^T x by the transposed forms."""
    N, D, H = 300, 200, 150
    x, w, dy = _matrix(N, D, torch.bfloat16, 1, 0.3), _matrix(H, D, torch.float32, 2, 0.3), _matrix(N, H, torch.bfloat16, 3, 0.3)
    xq, xt, wq, wt = am.q8_empty(N, D), am.q8_empty(D, N), am.q8_empty(H, D, True), am.q8_empty(D, H, True)
    dq, dt = am.q8_empty(N, H), am.q8_empty(H, N)
    am.q8_quantise(x, *xq, *xt)
    am.q8_quantise(w, *wq, *wt, tiles=True)
    am.q8_quantise(dy, *dq, *dt)
    y, dx, dw = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((N, H), (N, D), (H, D)))
    _product(xq, wq, y, tiles=True)
    _product(dq, wt, dx, tiles=True)
    _product(dt, xt, dw)
    # a code is off by 2^-4 of the value at most, both factors' by 2^-3 and a little: the
    # sum's error is below that part of the sum of magnitudes
    for out, p, q in ((y, x, w.t()), (dx, dy, w), (dw, dy.t(), x)):
        p, q = _f64(p), _f64(q)
        assert np.all(np.abs(_f64(out) - p @ q) <= (2.0 ** -3 + 2.0 ** -7) * (np.abs(p) @ np.abs(q)) + 2.0 ** -8 * np.abs(p @ q))


@BOTH
@pytest.mark.parametrize("stream", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,H", [(1, 1), (3, 16), (5, 100), (2, 128), (7, 129), (64, 768), (3, 1000), (2, 2048), (2, 5000),
                                 (3, 8192)])
def test_norm(N, H, stream, dtype):
    rng = np.random.default_rng(N + H)
    dev = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    o, gate, res = dev(N, H).to(dtype), dev(N, H).to(dtype), dev(N, H).to(stream)
    w = dict(w_post=dev(H), scale=dev(H), w_next=dev(H))
    want, got = (dict(res_out=torch.empty_like(res), y=torch.empty_like(o), rstd=torch.empty((N, 2), device="cuda"))
                 for _ in range(2))
    am.gated_norm_forward(res, o=o, gate=gate, **w, **want)
    codes, scales = _room(N, H)
    am.gated_norm_forward_q8(res, codes, scales, o=o, gate=gate, **w, **got)
    for k in want:  # what both calls write is the same
        assert torch.equal(want[k], got[k]), k
    alone, s2 = _room(N, H)
    am.gated_norm_forward_q8(res, alone, s2, o=o, gate=gate, **w, res_out=torch.empty_like(res))
    assert np.array_equal(_whole(alone), _whole(codes)) and torch.equal(s2.view(torch.uint8), scales.view(torch.uint8))
    raw = _whole(codes)
    assert np.all(raw[:, H:] == 0)
    y = gated.gated_norm_forward(_f64(res), o=_f64(o), gate=_f64(gate), **{k: _f64(v) for k, v in w.items()})[1]
    e = scales.view(torch.uint8).cpu().numpy()[:, :-(-H // 128)]
    want_e = q8.exponents(y)
    # (a largest value within 1e-5 of a power of two may fall on either side of it)
    near = np.abs(q8.exponents(y * (1 + 1e-5)).astype(int) - q8.exponents(y * (1 - 1e-5)).astype(int)) > 0
    assert np.all((e == want_e) | near)
    scale = q8.spread(e, y.shape)
    # half a step of a code: 2^-4 of it, and 2^-10 of a subnormal one; 1e-5 of the norm in 32 bits
    err = np.abs(q8.value(raw[:, :H]) * scale - y)
    assert np.all(err <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale) + 1e-5 * np.abs(y) + 1e-30)


def test_norm_of_the_stream_alone():
    res, w = torch.randn((9, 300), device="cuda"), torch.randn(300, device="cuda")
    y = torch.empty_like(res)
    am.gated_norm_forward(res, w_next=w, y=y)
    codes, scales = _room(9, 300)
    am.gated_norm_forward_q8(res, codes, scales, w_next=w)
    value, e = q8.quantise(_f64(y))
    assert np.array_equal(scales.view(torch.uint8).cpu().numpy()[:, :3], e)
    assert np.array_equal(q8.value(_whole(codes)[:, :300]), value)


def test_run_together_in_a_graph():
    """Norm, projection, recurrence and the norm behind it, as a block of a student runs."""
    T, B, H, heads = 70, 4, 256, 4
    dk = dv = H // heads
    N, cols = T * B, 3 * H + 2 * heads
    torch.manual_seed(1)
    res, w_next = torch.randn((N, H), device="cuda"), torch.ones(H, device="cuda")
    w = am.q8_empty(cols, H, True)
    am.q8_quantise(torch.randn((cols, H), device="cuda") * H ** -0.5, *w, tiles=True)
    lam = torch.full((heads,), -3.0, device="cuda")
    y, z = am.q8_empty(N, H), am.q8_empty(N, H)
    p, o = torch.empty((N, cols), dtype=torch.bfloat16, device="cuda"), torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(res)
    at = np.cumsum([0, H, H, H, heads, heads]).tolist()

    def block():
        am.gated_norm_forward_q8(res, *y, w_next=w_next)
        am.q8_matmul(*y, *w, p, tiles=True)
        am.gated_delta_forward(*[p[:, at[n]:at[n + 1]] for n in range(5)], lam, T, B, o, heads=heads)
        am.gated_norm_forward_q8(res, *z, o=o, w_post=w_next, w_next=w_next, res_out=out)

    block()
    torch.cuda.synchronize()
    from oracle import delta
    x = [_f64(p[:, at[n]:at[n + 1]]) for n in range(5)]
    ref = delta.gated_delta_forward(*x, _f64(lam), T, B, heads, heads)[0]
    assert np.abs(_f64(o) - ref).max() <= (2.0 ** -8 + 1e-4) * np.abs(ref).max()
    want = [t.clone() for t in (p, o, out, z[0].view(torch.uint8))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for _ in range(3):
        for t in (p, o, out):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (p, o, out, z[0].view(torch.uint8))):
            assert torch.equal(a, b)
