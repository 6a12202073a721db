"""AdamW step of many tensors: against the exact fp32 order bit for bit (weights,
bf16 copy, moments, 8-bit codes and scales) and against fp64.

Tolerance against fp64: m, v, the root, the quotient and the products of a step
round about ten times, 1e-6 of the step, and the weight itself once, 6e-8 of it."""

import numpy as np
import pytest
import torch

import oracle
from oracle import adamw
from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

OPT = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)


class Tensors:
    """Tensors of these sizes, `skew` elements into their allocations, with the
    same values kept on the host."""

    def __init__(self, sizes, bits, grad=torch.float32, skew=0, copy=True, seed=0, scale=1e-3):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits, self.host, self.dev = sizes, bits, [], []
        put = lambda a: self._at(torch.from_numpy(a).cuda(), skew)  # noqa: E731
        for k, n in enumerate(sizes):
            f = lambda s=1.0: (rng.standard_normal(n) * s).astype(np.float32)  # noqa: E731
            h = {"master": f(0.05), "grad": f(scale), "weight_decay": 0.01 * (k % 2)}
            d = {"master": put(h["master"]), "grad": self._at(torch.from_numpy(h["grad"]).cuda().to(grad), skew),
                 "weight_decay": h["weight_decay"]}
            h["grad"] = d["grad"].float().cpu().numpy()
            m, v = f(scale), f(scale) ** 2
            if bits == 32:
                h.update(m=m, v=v)
            else:
                z = np.zeros(n, np.int64)
                h["m"], h["m_scale"] = adamw.encode(m, z, 0)
                h["v"], h["v_scale"] = adamw.encode(np.sqrt(v), z, 1)
                d.update(m_scale=put(h["m_scale"]), v_scale=put(h["v_scale"]))
            d.update(m=put(h["m"]), v=put(h["v"]))
            if copy:
                d["weights_bf16"] = self._at(torch.zeros(n, dtype=torch.bfloat16, device="cuda"), skew)
            self.host.append(h)
            self.dev.append(d)

    @staticmethod
    def _at(t, skew):
        whole = torch.zeros(t.numel() + skew, dtype=t.dtype, device="cuda")
        whole[skew:] = t
        return whole[skew:]

    def expect(self, step, seed=0, grad_scale=None):
        for k, h in enumerate(self.host):
            c = adamw.coefficients(step=step, weight_decay=h["weight_decay"], **OPT)
            if self.bits == 32:
                m, v = h["m"], h["v"]
            else:
                r = adamw.decode(h["v"], h["v_scale"])
                with np.errstate(all="ignore"):
                    m, v = adamw.decode(h["m"], h["m_scale"]), r * r
            h["master"], m, v, r = adamw.step_f32(h["master"], h["grad"], m, v, c, grad_scale)
            if self.bits == 32:
                h.update(m=m, v=v)
            else:
                for_m, for_v = adamw.draws(m.size, k, seed)
                h["m"], h["m_scale"] = adamw.encode(m, for_m, 0)
                h["v"], h["v_scale"] = adamw.encode(r, for_v, 1)

    def compare(self):
        torch.cuda.synchronize()
        for k, (h, d) in enumerate(zip(self.host, self.dev)):
            for name in ("master", "m", "v") + (() if self.bits == 32 else ("m_scale", "v_scale")):
                got, want = d[name].cpu().numpy(), h[name]
                if got.dtype == np.float32:  # (NaN's payload is not fixed)
                    same = (got.view(np.uint32) == want.view(np.uint32)) | (np.isnan(got) & np.isnan(want))
                else:
                    same = (got == want) | (((got & 127) == 127) & ((want & 127) == 127))
                assert np.all(same), (k, name, np.flatnonzero(~same)[:5], got[~same][:5], want[~same][:5])
            if "weights_bf16" in d:
                got = d["weights_bf16"].view(torch.int16).cpu().numpy().view(np.uint16)
                np.testing.assert_array_equal(got, oracle.bf16_bits(h["master"]))


SIZES = [1, 3, 4, 5, 0, 255, 256, 257, 511, 1024, 2047, 2048, 2049, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("skew", [0, 1, 2, 3])
def test_bit_for_bit(bits, grad, skew):
    t = Tensors(SIZES, bits, grad, skew, copy=skew != 2, seed=skew)
    handle = am.AdamWTensors(t.dev)
    for step in (1, 2, 1000):
        am.adamw_apply(handle, step=step, seed=step, **OPT)
        t.expect(step, seed=step)
    t.compare()


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes(bits):
    rng = np.random.default_rng(1)
    t = Tensors([int(n) for n in rng.integers(0, 600, 131)], bits, seed=2)
    am.adamw_apply(am.AdamWTensors(t.dev), step=7, seed=0xFFFFFFFF, **OPT)
    t.expect(7, seed=0xFFFFFFFF)
    t.compare()


@pytest.mark.parametrize("bits", [32, 8])
def test_scaled_gradients_and_skipped_steps(bits):
    t = Tensors([300, 5000], bits)
    handle = am.AdamWTensors(t.dev)
    gs = torch.tensor([0.37], device="cuda")
    am.adamw_apply(handle, step=3, grad_scale=gs, **OPT)
    t.expect(3, grad_scale=np.float32(0.37))
    for bad in (float("inf"), float("-inf"), float("nan")):
        am.adamw_apply(handle, step=4, grad_scale=gs.fill_(bad), **OPT)
    t.compare()


@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_not_finite_stays_in_its_element(bits):
    t = Tensors([700], bits)
    for at, v in ((5, np.inf), (300, -np.inf), (301, np.nan)):
        t.host[0]["grad"][at] = v
        t.dev[0]["grad"][at] = float(v)
    handle = am.AdamWTensors(t.dev)
    for step in (5, 6):
        am.adamw_apply(handle, step=step, **OPT)
        t.expect(step)
    t.compare()
    assert int(torch.isnan(t.dev[0]["master"]).sum()) == 3


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e10])
def test_moments_of_any_magnitude(scale):
    t = Tensors([1000], 8, scale=scale, seed=3)
    handle = am.AdamWTensors(t.dev)
    for step in (1, 2):
        am.adamw_apply(handle, step=step, seed=step, **OPT)
        t.expect(step, seed=step)
    t.compare()


def test_against_64_bits():
    t = Tensors([5000], 32, copy=False)
    h = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in t.host[0].items()}
    am.adamw_apply(am.AdamWTensors(t.dev), step=10, **OPT)
    w, m, v = adamw.step_f64(h["master"], h["grad"], h["m"], h["v"], step=10,
                             weight_decay=h["weight_decay"], **OPT)
    moved = np.abs(w - h["master"])
    assert np.all(np.abs(t.dev[0]["master"].cpu().numpy() - w) <= 1e-6 * moved + 1.2e-7 * np.abs(w))
    np.testing.assert_allclose(t.dev[0]["m"].cpu().numpy(), m, rtol=1e-6, atol=1e-10)
    np.testing.assert_allclose(t.dev[0]["v"].cpu().numpy(), v, rtol=1e-6)


def test_8_bit_moments_follow_the_gradient():
    """Gradients of one size for 3000 steps, from moments a hundred times too
    large: the second moment decays to theirs, which codes rounded to nearest
    would never leave.  Rounding a root r = 1 moves it by a unit of up to 1 / 8 with
    probability |change| / unit, a variance of up to 0.0005 / 8 a step against a
    decay of 0.001 a step: 18 % an element (five of it bound all 4096), and 1 +
    0.0005 / 8 / 0.001 = 1.06 for the mean of the second moment."""
    n = 4096
    d = {"master": torch.zeros(n, device="cuda"), "grad": torch.empty(n, device="cuda"),
         "m": torch.zeros(n, dtype=torch.uint8, device="cuda"), "v": torch.zeros(n, dtype=torch.uint8, device="cuda"),
         "m_scale": torch.zeros(16, device="cuda"), "v_scale": torch.zeros(16, device="cuda")}
    handle = am.AdamWTensors([d])
    gen = torch.Generator(device="cuda").manual_seed(5)
    for step in range(1, 12001):
        d["grad"].normal_(generator=gen)
        if step <= 20:
            d["grad"].mul_(100.0)
        am.adamw_apply(handle, step=step, seed=step, **OPT)
    r = d["v"].view(torch.float8_e4m3fn).float() * d["v_scale"].repeat_interleave(256)
    assert 0.9 < float((r * r).mean()) < 1.2
    assert 0.1 < float(r.min()) and float(r.max()) < 1.9


def test_elements_past_32_bits():
    """A tensor of more than 2^31 elements: its last ones as by themselves."""
    n = (1 << 31) + 4096 + 5
    d = {k: torch.zeros(n, device="cuda") for k in ("master", "m", "v")}
    d["grad"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(4096, device="cuda").to(torch.bfloat16)
    d["grad"][-4096:] = tail
    am.adamw_apply(am.AdamWTensors([d]), step=1, **OPT)
    s = {k: torch.zeros(4096, device="cuda") for k in ("master", "m", "v")}
    s["grad"] = tail
    am.adamw_apply(am.AdamWTensors([s]), step=1, **OPT)
    for k in ("master", "m", "v"):
        assert torch.equal(d[k][-4096:], s[k]) and not d[k][:8192].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_large_step_is_the_small_ones(bits):
    """More than the caches hold (accesses go past them): the first elements as by
    themselves."""
    n, few = 45_000_001, 256 * 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    kind = torch.float32 if bits == 32 else torch.uint8
    d = {k: torch.randn(n, device="cuda", generator=gen) for k in ("master", "grad")}
    d.update({k: torch.zeros(n, dtype=kind, device="cuda") for k in ("m", "v")})
    d["weights_bf16"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    if bits == 8:
        d.update({k: torch.zeros(am.adamw_scales(n), device="cuda") for k in ("m_scale", "v_scale")})
    s = {k: t[:few // 256 if "scale" in k else few].clone() for k, t in d.items()}
    for step in (1, 2):
        am.adamw_apply(am.AdamWTensors([d]), step=step, seed=step, **OPT)
        am.adamw_apply(am.AdamWTensors([s]), step=step, seed=step, **OPT)
    for k, t in s.items():
        assert torch.equal(d[k][:t.numel()], t), k


def test_from_a_graph_and_on_a_stream():
    t, u = Tensors([300, 70001], 8), Tensors([300, 70001], 8)
    a, b = am.AdamWTensors(t.dev), am.AdamWTensors(u.dev)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        am.adamw_apply(a, step=9, seed=4, **OPT)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            am.adamw_apply(b, step=9, seed=4, **OPT)
        s.synchronize()
        for x, y in zip(t.dev, u.dev):
            assert all(torch.equal(x[k], y[k]) for k in x if isinstance(x[k], torch.Tensor))
