"""Matrices in 8 bits where rows are not finite, and how far a product is from its size."""

import numpy as np
import pytest
import torch

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
