"""The norms between two blocks over more rows than there are compute units to hold
a workgroup each, so that waves share their SIMDs: every width's kernel, against
the fp64 oracle.  Tolerances as in test_gpu_gated_norm."""

import pytest
import torch

from test_gpu_gated_norm import BF16, F32, _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("N,H", [(5000, 2), (3900, 10), (3000, 18), (4096, 64), (3967, 182), (4000, 252), (3100, 255),
                                 (3000, 500), (2600, 767), (2500, 1022), (2200, 1535), (2100, 2046), (2100, 3069),
                                 (2100, 4094), (2050, 8190)])
def test_many_rows_of_any_width(N, H, dtype, stream):
    _check(*_inputs(N, H, dtype, stream, seed=N + H))
