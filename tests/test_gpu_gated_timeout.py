"""A wait of the gated recurrence that ran out: the flag, the check and the zeros in
place of gradients.  No kernel is made to wait: the flag (last word of the
workspace's first 8 KiB) is set between the calls, as such a wait sets it."""

import pytest
import torch

from paper_1904_10584_amd import binding as am
from test_gpu_gated_recurrence import Case

pytestmark = pytest.mark.gpu

# one tile, tiles in turn, linked tiles; equal lengths and others
SHAPES = [(1, 4, 96, None), (64, 3, 96, None), (200, 3, 96, None), (9000, 1, 96, None), (70, 3, 96, [70, 33, 1]),
          (200, 4, 96, [200, 33, 1, 0]), (5000, 3, 96, [5000, 700, 0])]


def _flag(ws):
    return ws[8188:8192].view(torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,H,lengths", SHAPES)
def test_a_pass_that_timed_out_leaves_zero_gradients(T, B, H, lengths, dtype):
    c = Case(T, B, H, dtype, lengths, pad=3, seed=31)
    c.forward()  # (into a workspace of 0xFF bytes)
    am.workspace_check(c.ws)
    want = c.backward()
    am.workspace_check(c.ws)
    _flag(c.ws).fill_(1)
    dproj = torch.full_like(c.proj, 7.0)
    dlam, dh0 = torch.full((H,), 7.0, device="cuda"), torch.full((B, H), 7.0, device="cuda")
    am.gated_recurrence_backward(*c.cols(c.proj), c.lam, T, B, c.dh, c.ws, *c.cols(dproj), dlam, lengths=lengths,
                                 dhT=c.dhT, dh0=dh0)
    with pytest.raises(am.AmError) as e:
        am.workspace_check(c.ws)
    assert e.value.status == am.ETIMEOUT
    assert not any(t.any() for t in (*c.cols(dproj), dlam, dh0))
    assert torch.all(dproj[:, :3] == 7)
    # the next forward call clears it
    ws = c.ws
    h, hT = torch.empty((c.N, H), dtype=dtype, device="cuda"), torch.empty((B, H), device="cuda")
    am.gated_recurrence_forward(*c.cols(c.proj), c.lam, T, B, h, ws, lengths=lengths, h0=c.h0, hT=hT, train=True)
    am.workspace_check(ws)
    assert all(torch.equal(a, b) for a, b in zip(c.backward(), want))
    am.workspace_check(ws)


@pytest.mark.parametrize("T,B,H,lengths", [(9000, 1, 96, None), (70, 3, 96, [70, 33, 1])])
def test_scoring_clears_the_flag_too(T, B, H, lengths):
    c = Case(T, B, H, lengths=lengths, seed=32)
    c.forward(train=False)
    am.workspace_check(c.ws)


def test_a_workspace_that_may_be_empty_is_not_written():
    """One frame a sequence needs none; one that is given stays as it is."""
    c = Case(1, 4, 96, seed=33)
    ws = torch.full((16384,), 0xFF, dtype=torch.uint8, device="cuda")
    h = torch.empty((4, 96), dtype=torch.bfloat16, device="cuda")
    am.gated_recurrence_forward(*c.cols(c.proj), c.lam, 1, 4, h, ws)
    assert torch.all(ws == 0xFF)


@pytest.mark.parametrize("bits", [32, 8])
def test_the_student_keeps_its_weights_where_the_loss_is_not_finite(bits):
    from examples.gated_student import GatedStudent
    from paper_1904_10584_amd import synth
    s = GatedStudent(2, 24, 48, 100, 20, 3, 4, bits=bits)
    x = torch.from_numpy(synth.features(60, 24)).cuda()
    idx, prob = (torch.from_numpy(v).cuda() for v in synth.teacher_targets(60, 100, 4, 0.95))
    s.step(x, idx, prob)
    s.check()
    before = {k: v.clone() for k, v in s.master.items()}
    bad = x.clone()
    bad[7, 5] = float("nan")
    assert not torch.isfinite(s.step(bad, idx, prob))
    assert all(torch.equal(v, s.master[k]) for k, v in before.items())
    assert torch.isfinite(s.step(x, idx, prob))
    assert not any(torch.equal(v, s.master[k]) for k, v in before.items())
    _flag(s.rec_ws[1]).fill_(1)
    with pytest.raises(am.AmError):
        s.check()
