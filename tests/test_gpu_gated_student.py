"""The gated student of examples/gated_student.py: its gradients against
differentiation in fp64, training with 32-bit and with 8-bit moments, and frame
by frame against whole sequences."""

import math

import pytest
import torch

from gpu_util import assert_close
from paper_1904_10584_amd import synth

pytestmark = pytest.mark.gpu

L, D, H, C, K = 2, 24, 48, 100, 4


def _student(T, B, lengths=None, **kw):
    from examples.gated_student import GatedStudent
    return GatedStudent(L, D, H, C, T, B, K, lengths=lengths, **kw)


def _batch(N):
    x = torch.from_numpy(synth.features(N, D)).cuda()
    idx, prob = (torch.from_numpy(v).cuda() for v in synth.teacher_targets(N, C, K, 0.95))
    return x, idx, prob


def _reference(p, x, idx, prob, T, B, lengths):
    """The student's loss by definition, in fp64 on the CPU."""
    lens = lengths or [T] * B
    norm = lambda v: v * torch.rsqrt(v.pow(2).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    res = x @ p["Win"].t()
    y = norm(res) * p["w0"]
    for l in range(L):
        a, r, i = (y @ p[f"Wp{l}"].t()).split(H, 1)
        rate = 8.0 * torch.nn.functional.softplus(p[f"lam{l}"]) * torch.sigmoid(r)
        u = torch.sqrt(-torch.expm1(-2 * rate)) * torch.sigmoid(i) * a
        h, out, at = torch.zeros(B, H, dtype=torch.float64), [], 0
        for t in range(T):
            nb = sum(n > t for n in lens)
            h = torch.exp(-rate[at:at + nb]) * h[:nb] + u[at:at + nb]
            out.append(h)
            at += nb
        z = torch.cat(out) * torch.nn.functional.silu(y @ p[f"Wg{l}"].t())
        res = res + p[f"scale{l}"] * p[f"post{l}"] * norm(z)
        y = norm(res) * p[f"next{l}"]
    logp = torch.log_softmax(y @ p["Wo"].t() + p["bo"], 1)
    return -(prob * logp.gather(1, idx)).sum(1).mean()


@pytest.mark.parametrize("T,B,lengths", [(20, 3, None), (70, 4, [70, 66, 31, 2])])
def test_gradients_are_the_definitions(T, B, lengths):
    """fp32 throughout: the products' sums of up to 100 terms and the recurrence's
    err by about 1e-5 of their size; 1e-4, as the framework's other fp32 paths."""
    s = _student(T, B, lengths, dtype=torch.float32)
    x, idx, prob = _batch(s.N)
    before = {k: v.double().cpu().requires_grad_() for k, v in s.master.items()}
    loss = s.step(x, idx, prob)
    ref = _reference(before, x.double().cpu(), idx.long().cpu(), prob.double().cpu(), T, B, lengths)
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) <= 1e-4 * float(ref.detach())
    for k, v in before.items():
        assert_close(k, s.grads[k].cpu().numpy(), v.grad.numpy(), 1e-4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns(bits, dtype):
    """A fixed batch of 200 frames, random inputs and Zipf targets: from about ln C
    times the targets' mass, to below two thirds of it in 150 steps."""
    s = _student(25, 8, dtype=dtype, bits=bits)
    batch = _batch(200)
    first = float(s.step(*batch))
    assert abs(first - 0.95 * math.log(C)) < 0.8
    for _ in range(149):
        last = s.step(*batch)
    assert float(last) < 2 / 3 * first, (first, float(last))


def test_frame_by_frame_is_the_whole():
    T, B = 30, 5
    s = _student(T, B, dtype=torch.float32)
    x, _, _ = _batch(T * B)
    want = s.forward(x)
    states = torch.zeros((L, B, H), device="cuda")
    got = torch.cat([s.stream(states, x[t * B:(t + 1) * B]) for t in range(T)])
    assert_close("logits", got.cpu().numpy(), want.cpu().numpy(), 1e-4)
