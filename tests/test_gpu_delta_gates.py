"""The gated delta rule's gates at their ends, against the fp64 oracle."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close
from test_gpu_delta import BF16_TOL, F32_TOL, Case, _f64

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
NAMES = ("o", "sT", "dq", "dk", "dv", "dr", "db", "dlam", "ds0")


@BOTH
@pytest.mark.parametrize("T,lengths", [(130, None), (1, None), (70, [70, 3])])
def test_shut_gates_of_a_rate_past_32_bits(T, lengths, dtype):
    """c softplus(lam) = 2.4e39 times a sigmoid of e^-200: nothing decays."""
    c = Case(T, 2, 2, 32, 32, dtype, seed=9, lam=(3e38, 3e38), lengths=lengths)
    c.cols(c.proj)[3].fill_(-200.0)
    got, ref = c.forward() + c.backward(), c.oracle()
    tol = BF16_TOL if dtype == torch.bfloat16 else F32_TOL
    for name, g, w in zip(NAMES, got, ref):
        assert np.isfinite(_f64(g)).all(), name
        if name in ("dr", "dlam"):  # (e^-200 of the rest)
            assert np.abs(_f64(g)).max() < 1e-30 and np.abs(w).max() < 1e-30, name
        else:
            assert_close(name, _f64(g), w, tol if g.dtype == dtype else F32_TOL)
    o, sT = c.forward(train=False)
    assert_close("o, serving", _f64(o), ref[0], tol)
    assert_close("sT, serving", _f64(sT), ref[1], F32_TOL)
