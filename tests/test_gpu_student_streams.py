"""The student of examples/gated_student.py frame by frame where its streamed products
are split and those of training are not."""

import pytest
import torch

from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu


def test_a_wide_student_with_8_bit_products_streams():
    """Frames by themselves are the sequence: in bf16 with 8-bit products their sums
    differ in their order alone, which moves a few roundings to bf16 and to e4m3: 5 % of
    the logits' size, as one product of two operands that differ in every rounding."""
    from examples.gated_student import GatedStudent
    T, B, D, H, C = 3, 700, 24, 4096, 60
    s = GatedStudent(1, D, H, C, T, B, 4, projections=8)
    rows = (H, 3 * H)
    assert max(am.q8_matmul_workspace_bytes(T * B, n, H) for n in rows) == 0
    x = torch.randn((T * B, D), device="cuda")
    want = s.forward(x).double().view(T, B, C)
    for n in (1, 64):  # a few of the sequences, whose products are split
        assert max(am.q8_matmul_workspace_bytes(n, m, H) for m in rows) > s.q8_ws.numel()
        states = torch.zeros((1, n, H), device="cuda")
        got = torch.stack([s.stream(states, x.view(T, B, D)[t, :n]) for t in range(T)]).double()
        assert float((got - want[:, :n]).norm() / want[:, :n].norm()) <= 0.05
