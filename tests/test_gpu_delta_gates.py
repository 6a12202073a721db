"""Gradients of the gated delta rule's gates against the fp64 oracle, where they are
small: decays from a few percent to e^-70 a frame, gates nearly open or nearly shut.

The gradient of log a_t carries the factor a_t.  a_t = e^-x with x = c softplus(lam)
sigm(r) up to 87, which is off by 2^-22 of itself at most (softplus, sigm and two
products in 32 bits), so a_t by 87 2^-22 = 2.1e-5; what it multiplies are products and
sums in 32 bits, 1.2e-5.  (From x = 126 log 2 = 87.3 on, a_t is below the normal 32-bit
floats, and the hardware's exponential gives 0: what is there, less than 2^-126 of the
other frames' size, may be lost.)  Together below 1e-4, the bound of this library's fp32 outputs;
with bf16 inputs dO and U meet with U in 16 bits, 2^-17, which leaves that as it is, and
one rounding, 2^-8, of dr.  Every frame's gradient is held to that bound at its own decay:
what is compared is dr / a_t.  dlam is a sum over frames: it is held to 1e-4 of the sum of
its terms' magnitudes."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close
from test_gpu_delta import BF16_TOL, F32_TOL, Case, _f64

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
C = 8.0
NAMES = ("o", "sT", "dq", "dk", "dv", "dr", "db", "dlam", "ds0")


def _gates(c):
    """c softplus(lam), sigm(r) and sigm(-r) by frame and head, in fp64."""
    rate, r = C * np.logaddexp(0, _f64(c.lam)), _f64(c.cols(c.proj)[3])
    return rate, 1 / (1 + np.exp(-r)), 1 / (1 + np.exp(r))


def _check(c, weight):
    """dr times weight, and dlam, against the oracle; every output finite."""
    got, ref = c.forward() + c.backward(), c.oracle()
    for g in got:
        assert np.isfinite(_f64(g)).all()
    dr, want = _f64(got[5]) * weight, ref[5] * weight
    tol = F32_TOL if c.dtype == torch.float32 else BF16_TOL
    # (dr is rate e sigm(r) sigm(-r) of the gradient -e of log a, dlam the sum of c e sigm(r) sigm(lam))
    rate, sr, rest = _gates(c)
    lost = np.where(rate * sr > 126 * np.log(2.0), np.abs(want), 0.0)
    assert np.all(np.abs(dr - want) <= tol * np.abs(want).max() + lost), np.abs(dr - want).max() / np.abs(want).max()
    terms = np.abs(ref[5] / (rate * rest)).sum(0) * C / (1 + np.exp(-_f64(c.lam)))
    off = np.abs(_f64(got[7]) - ref[7])
    assert np.all(off <= F32_TOL * terms), (off / terms).max()


@BOTH
@pytest.mark.parametrize("lam", [-3.0, 0.0, 1.0, 2.0, 3.0, 5.0, 8.0, 12.0, 16.0])
def test_decays_of_any_strength(lam, dtype):
    c = Case(130, 2, 2, 32, 32, dtype, seed=int(lam) + 40, lam=(lam, lam + 0.01))
    c.cols(c.proj)[3].mul_(0.3)
    rate, sr, _ = _gates(c)
    _check(c, np.exp(rate * sr))


@BOTH
@pytest.mark.parametrize("T,B,heads,keys,dk,dv,lengths", [
    (1, 3, 2, 2, 64, 64, None), (64, 1, 1, 1, 64, 64, None), (65, 2, 4, 1, 24, 40, None),
    (200, 5, 4, 2, 100, 33, [200, 129, 128, 1, 0]), (1700, 2, 1, 1, 40, 24, [1700, 513]), (90, 1, 1, 1, 128, 128, None)])
def test_strong_decays_in_every_form(T, B, heads, keys, dk, dv, lengths, dtype):
    """Chunks, ragged ends, heads that share keys, wide heads, segments."""
    c = Case(T, B, heads, dk, dv, dtype, keys=keys, lengths=lengths, seed=T + dk, lam=(4.0, 4.01))
    c.cols(c.proj)[3].mul_(0.3)
    rate, sr, _ = _gates(c)
    _check(c, np.exp(rate * sr))


@BOTH
def test_frames_that_forget_among_frames_that_keep(dtype):
    """Every fifth frame forgets by e^-20 or so, the others by 0.1 %."""
    c = Case(130, 2, 2, 32, 32, dtype, seed=6, lam=(4.0, 4.01))
    r = c.cols(c.proj)[3]
    r.mul_(0.3).sub_(10.0)
    r[::5] += 10.0
    rate, sr, rest = _gates(c)
    _check(c, np.exp(rate * sr) / (sr * rest))


@BOTH
@pytest.mark.parametrize("what", ["two keys", "zero rows", "shut"])
def test_edges(what, dtype):
    """Repeated keys, rows without a length, gates that write nothing."""
    c = Case(130, 2, 2, 32, 32, dtype, seed=3)
    q, k, v, r, b = c.cols(c.proj)
    if what == "two keys":
        k[::2] = k[:1].clone()
        k[1::2] = k[1:2].clone()
        b.fill_(30.0)
    elif what == "zero rows":
        q[5:9], k[3:70], v[60:] = 0, 0, 0
    else:
        b.fill_(-200.0)
    _check(c, 1.0)


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


@BOTH
@pytest.mark.parametrize("gate", [5.0, 8.0, 12.0, 16.0, 30.0, 60.0])
def test_gates_nearly_open(gate, dtype):
    """r and b of 5 to 60: the gradients carry sigm(-r) and sigm(-b), as small as e^-60,
    and are held to their bounds beside them."""
    c = Case(130, 2, 2, 32, 32, dtype, seed=int(gate))
    r, b = c.cols(c.proj)[3:]
    for t in (r, b):
        t.mul_(0.3).add_(gate)
    got, ref = c.forward() + c.backward(), c.oracle()
    tol = F32_TOL if dtype == torch.float32 else BF16_TOL
    for name, t, n in (("dr", r, 5), ("db", b, 6)):
        x = np.exp(_f64(t))  # 1 / sigm(-t), but for 1
        want = ref[n] * x
        assert np.abs(_f64(got[n]) * x - want).max() <= tol * np.abs(want).max(), name


@BOTH
def test_more_heads_of_a_key_than_a_workgroup_has_threads(dtype):
    """Chunks that a sequence does not reach have no part in dlam, of any head."""
    c = Case(66, 2, 600, 4, 4, dtype, keys=1, lengths=[65, 3], seed=4)
    c.check()
