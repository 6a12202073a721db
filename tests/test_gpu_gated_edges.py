"""Gated recurrence where its two passes are called differently and where a
sequence has no frames.  Tolerances as in test_gpu_gated_recurrence."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close
from paper_1904_10584_amd import binding as am
from test_gpu_gated_recurrence import BF16_TOL, F32_TOL, Case

pytestmark = pytest.mark.gpu


def _one_element_in(*shape, dtype=torch.bfloat16):
    """A contiguous tensor that starts one element into its buffer."""
    n = int(np.prod(shape))
    return torch.full((n + 1,), float("nan"), dtype=dtype, device="cuda")[1:].view(*shape)


@pytest.mark.parametrize("odd_forward,odd_backward", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("H,lengths", [(64, [200, 10]), (38, [200, 130, 129, 10, 5, 2]), (130, [300, 10, 10]),
                                       (64, [700, 10]), (38, [1500, 1400, 70, 1])])
def test_one_pass_on_odd_addresses(H, lengths, odd_forward, odd_backward):
    """bf16 tensors on odd elements in one pass and even ones in the other: each
    pass groups channels in its own way, and the backward pass takes nothing from
    the workspace (0xFF bytes before) that the forward pass did not write."""
    T, B = max(lengths), len(lengths)
    c = Case(T, B, H, torch.bfloat16, lengths, seed=H)
    c.forward()  # (makes the workspace)
    c.ws.fill_(0xFF)
    new = lambda odd: _one_element_in(c.N, H) if odd else torch.empty((c.N, H), dtype=c.dtype, device="cuda")  # noqa: E731
    h, hT = new(odd_forward), torch.empty((B, H), device="cuda")
    am.gated_recurrence_forward(*c.cols(c.proj), c.lam, T, B, h, c.ws, lengths=lengths, h0=c.h0, hT=hT, train=True)
    dh, dx, dr, di = (new(odd_backward) for _ in range(4))
    dh.copy_(c.dh)
    dlam, dh0 = torch.empty(H, device="cuda"), torch.empty((B, H), device="cuda")
    am.gated_recurrence_backward(*c.cols(c.proj), c.lam, T, B, dh, c.ws, dx, dr, di, dlam, lengths=lengths,
                                 dhT=c.dhT, dh0=dh0)
    names = ("h", "hT", "dx", "dr", "di", "dlam", "dh0")
    for name, g, ref in zip(names, (h, hT, dx, dr, di, dlam, dh0), c.oracle()):
        assert_close(name, g.float().cpu().numpy(), ref, BF16_TOL if g.dtype == torch.bfloat16 else F32_TOL)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [[70, 20, 0], [700, 0, 0], [5, 0]])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_states_of_a_sequence_without_frames_stay_its_own(value, lengths, dtype):
    """The last sequence has no frames: whatever its states hold leaves as they
    are, and nothing else sees them."""
    T, B, H = max(lengths), len(lengths), 40
    c = Case(T, B, H, dtype, lengths, seed=21)
    ref = c.oracle()
    c.h0[-1], c.dhT[-1] = value, value
    got = c.forward() + c.backward()
    names = ("h", "hT", "dx", "dr", "di", "dlam", "dh0")
    for name, g, r in zip(names, got, ref):
        g = g.float().cpu().numpy()
        if name in ("hT", "dh0"):
            assert np.array_equal(g[-1], np.full(H, value, np.float32), equal_nan=True), name
            g, r = g[:-1], r[:-1]
        assert_close(name, g, r, BF16_TOL if dtype == torch.bfloat16 and name in ("h", "dx", "dr", "di") else F32_TOL)
