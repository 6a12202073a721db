"""Matrices in 8 bits where rows are not finite, and how far a product is from its size."""

import numpy as np
import pytest
import torch

from oracle import q8
from test_gpu_q8 import _room, _whole
from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H", [1, 100, 129, 250, 1000, 2049, 5000])
@pytest.mark.parametrize("bad", [NAN, float("inf")])
def test_norm_of_rows_that_are_not_finite(bad, H, dtype):
    """Their codes are NaN, the zeros behind them zeros, and the other rows' as without them."""
    torch.manual_seed(H)
    o, gate, res = (torch.randn((5, H), device="cuda") for _ in range(3))
    o, gate = o.to(dtype), gate.to(dtype)
    w = dict(w_post=torch.randn(H, device="cuda"), scale=torch.randn(H, device="cuda"), w_next=torch.randn(H, device="cuda"))
    want = _room(5, H)
    am.gated_norm_forward_q8(res, *want, o=o, gate=gate, **w, res_out=torch.empty_like(res))
    res[1, 0], o[3, H - 1] = bad, bad
    codes, scales = _room(5, H)
    am.gated_norm_forward_q8(res, codes, scales, o=o, gate=gate, **w, res_out=torch.empty_like(res))
    raw, clean = _whole(codes), _whole(want[0])
    assert np.all(raw[:, H:] == 0)
    for row in (0, 2, 4):
        assert np.array_equal(raw[row], clean[row])
        assert torch.equal(scales[row].view(torch.uint8), want[1][row].view(torch.uint8))
    for row in (1, 3):
        assert np.any((raw[row, :H] & 0x7F) == 0x7F)


def test_quantise_more_tiles_than_a_launch_has():
    """2^24 tiles of 256 threads: the ends and a part of the middle are those of the same
    rows by themselves."""
    rows = (1 << 31) - 1
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda")
    for at in range(0, rows, 1 << 28):
        x[at:at + (1 << 28)].normal_()
    codes, scales = am.q8_empty(1, rows)
    am.q8_quantise(x, codes_t=codes, scales_t=scales)
    for first in (0, 128 << 20, 128 * ((1 << 24) - 5)):
        part = x[first:first + 128 * 8]
        one, e = am.q8_empty(1, part.shape[0])
        am.q8_quantise(part, codes_t=one, scales_t=e)
        at = slice(first, first + part.shape[0])
        assert torch.equal(codes.view(torch.uint8)[:, at], one.view(torch.uint8)), first
        blocks = -(-part.shape[0] // 128)
        assert torch.equal(scales.view(torch.uint8)[:, first // 128:first // 128 + blocks], e.view(torch.uint8)[:, :blocks])


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("M,N,K", [(64, 256, 128), (64, 2304, 768), (512, 384, 4096), (300, 500, 16384), (768, 768, 16384),
                                   (2304, 768, 4099)])
def test_product_is_its_rounding_off(M, N, K, tiles):
    """The error of an output whose terms cancel, relative to the outputs' size in the
    root mean square.  Rounding to bf16 is evenly spread over half a step of at most 2^-8
    of a value: 2^-8 / sqrt(3) = 2.26e-3.  The matrix cores' sums of 128 products were
    found 2^-13.4 of the sum of magnitudes off in the root mean square at worst (products
    over the codes' whole range); of normal factors that sum is 128 2 / pi, and a block's
    own size sqrt(128): 6.7e-4, however many blocks are added.  Together 2.93e-3 at most."""
    torch.manual_seed(K)
    factors = [torch.randn((n, K), device="cuda") for n in (M, N)]
    a, b = am.q8_empty(M, K), am.q8_empty(N, K, tiles)
    am.q8_quantise(factors[0], *a)
    am.q8_quantise(factors[1], *b, tiles=tiles)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    am.q8_matmul(*a, *b, out, tiles=tiles,
                 ws=torch.empty(am.q8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda"))
    x, y = (q8.value(m[0].view(torch.uint8).cpu().numpy()) *
            q8.spread(m[1].view(torch.uint8).cpu().numpy()[:, :-(-K // 128)], m[0].shape, t) for m, t in ((a, False), (b, tiles)))
    want = x @ y.T
    off = np.sqrt(np.mean((out.float().cpu().numpy().astype(np.float64) - want) ** 2) / np.mean(want ** 2))
    assert off <= 2.93e-3, off
