"""Gated delta rule: forward and backward against the fp64 oracle.

Tolerances: products, states and sums are held in 32 bits.  A product over up to 128
columns and 64 frames with terms of like size is off by (128 + 64) 2^-24 of that size at
most, 1.2e-5; a state carries what it was off for the few frames that it remembers (the
decays of these cases: a few tens), which the next chunks' products see again: 1e-4, the
bound of every fp32 output of this library.  A bf16 output adds one rounding, half a step
or 2^-8 of the value: 2^-8 + 1e-4.

dq and dk are t - u (u t), what is left of the gradient t of a vector of unit length u
without its part along u.  Both terms are sums of dk products in 32 bits and are off by
2^-20 of t at most (a few units of 2^-24, the length's among them), whatever is left of
them: with one column that is the share of eps alone, 1e-6 of t.  So 2^-20 of the largest
t is added to their bound."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close
from oracle import delta
from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

F32_TOL = 1e-4
BF16_TOL = 2.0 ** -8 + F32_TOL
NAN = float("nan")


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


class Case:
    """Inputs on the GPU, columns of one matrix with `pad` columns before them."""

    def __init__(self, T, B, heads, dk, dv, dtype=torch.bfloat16, keys=None, lengths=None, pad=0, seed=0,
                 lam=(-6.0, -1.0)):
        rng = np.random.default_rng(seed)
        self.keys = keys or heads
        self.T, self.B, self.heads, self.dk, self.dv, self.lengths, self.dtype = T, B, heads, dk, dv, lengths, dtype
        self.N = T * B if lengths is None else int(sum(lengths))
        self.at = np.cumsum([pad, self.keys * dk, self.keys * dk, heads * dv, heads, heads]).tolist()
        dev = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
        self.proj = dev(self.N, self.at[-1] + pad).to(dtype)
        self.lam = torch.from_numpy(rng.uniform(*lam, heads).astype(np.float32)).cuda()
        self.s0, self.dsT = dev(B, heads, dk, dv), dev(B, heads, dk, dv)
        self.do = dev(self.N, heads * dv).to(dtype)

    def cols(self, t):
        return [t[:, self.at[n]:self.at[n + 1]] for n in range(5)]

    @staticmethod
    def _given(what, own):
        return own if what is True else None if what is False else what

    @property
    def sizes(self):
        return dict(heads=self.heads, key_heads=self.keys)

    def forward(self, s0=True, sT=None, train=True, **kw):
        need = am.gated_delta_workspace_bytes(self.T, self.B, dk=self.dk, dv=self.dv, dtype=self.dtype,
                                              lengths=self.lengths, train=train, **self.sizes)
        self.ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
        o = torch.full((self.N, self.heads * self.dv), NAN, dtype=self.dtype, device="cuda")
        sT = torch.full_like(self.s0, NAN) if sT is None else sT
        am.gated_delta_forward(*self.cols(self.proj), self.lam, self.T, self.B, o, self.ws, lengths=self.lengths,
                               s0=self._given(s0, self.s0), sT=sT, train=train, **self.sizes, **kw)
        return o, sT

    def backward(self, s0=True, dsT=True, ds0=None, **kw):
        dproj = torch.full_like(self.proj, NAN)
        dlam = torch.full((self.heads,), NAN, device="cuda")
        ds0 = torch.full_like(self.s0, NAN) if ds0 is None else ds0
        am.gated_delta_backward(*self.cols(self.proj), self.lam, self.T, self.B, self.do, self.ws, *self.cols(dproj),
                                dlam, lengths=self.lengths, s0=self.s0 if s0 else None,
                                dsT=self._given(dsT, self.dsT), ds0=ds0, **self.sizes, **kw)
        return (*self.cols(dproj), dlam, ds0)

    def oracle(self, s0=True, dsT=True):
        x = [_f64(t) for t in (*self.cols(self.proj), self.lam)]
        n = (self.T, self.B, self.heads, self.keys)
        o, sT, cache = delta.gated_delta_forward(*x, *n, self.lengths, _f64(self.s0) if s0 else None)
        back = delta.gated_delta_backward(*x, *n, _f64(self.do), cache, self.lengths, _f64(self.dsT) if dsT else None)
        self.along = dict(zip(("dq", "dk"), cache["along"]))
        return (o, sT) + back

    def close(self, name, g, ref):
        if g.numel():
            tol = BF16_TOL if g.dtype == torch.bfloat16 else F32_TOL
            if name in self.along:
                tol += 2.0 ** -20 * self.along[name] / max(float(np.sqrt(np.mean(ref * ref))), 1e-300)
            assert_close(name, _f64(g), ref, tol)

    def check(self, s0=True, dsT=True):
        got = self.forward(s0) + self.backward(s0, dsT)
        for name, g, ref in zip(("o", "sT", "dq", "dk", "dv", "dr", "db", "dlam", "ds0"), got, self.oracle(s0, dsT)):
            self.close(name, g, ref)


BOTH = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("T,B,heads,dk,dv", [
    (1, 1, 1, 1, 1), (1, 5, 3, 64, 64), (2, 3, 2, 8, 8), (15, 2, 2, 16, 48), (16, 1, 1, 32, 32), (17, 2, 1, 33, 31),
    (63, 2, 2, 64, 64), (64, 2, 2, 64, 64), (65, 2, 1, 64, 64), (64, 1, 2, 128, 128), (129, 1, 1, 128, 64),
    (130, 1, 2, 64, 128), (200, 2, 1, 65, 65), (100, 1, 1, 127, 17), (70, 1, 1, 3, 128), (81, 2, 2, 96, 100)])
def test_against_oracle(T, B, heads, dk, dv, dtype):
    Case(T, B, heads, dk, dv, dtype, seed=T + dk + dv).check()


@BOTH
@pytest.mark.parametrize("heads,keys", [(4, 1), (4, 2), (6, 3)])
def test_heads_that_share_keys(heads, keys, dtype):
    Case(70, 2, heads, 24, 40, dtype, keys=keys, seed=heads + keys).check()
    Case(70, 1, heads, 72, 8, dtype, keys=keys, seed=heads).check()


@BOTH
@pytest.mark.parametrize("lengths", [[5], [1, 0], [0, 0, 0], [7, 7, 3, 1, 0], [65, 64, 64, 63, 1],
                                     [200, 130, 129, 128, 127, 64, 8, 2], [150] + [1] * 40])
def test_ragged(lengths, dtype):
    Case(max(max(lengths), 1) + 2, len(lengths), 2, 20, 36, dtype, lengths=lengths, seed=len(lengths)).check()


@BOTH
@pytest.mark.parametrize("pad", [1, 2, 3, 8])
def test_columns_at_any_offset(pad, dtype):
    Case(70, 2, 2, 64, 64, dtype, pad=pad, seed=pad).check()
    Case(66, 2, 1, 23, 41, dtype, pad=pad, seed=pad).check()


# heads that fill the chip between them go through all chunks in one piece
@BOTH
@pytest.mark.parametrize("heads,dk,dv", [(180, 16, 24), (90, 70, 66)])
def test_many_heads(heads, dk, dv, dtype):
    c = Case(260, 4, heads // 2, dk, dv, dtype, keys=heads // 2, lengths=[260, 200, 129, 3], seed=heads)
    c.check()
    o, sT = c.forward()
    again = c.forward(train=False)
    assert torch.equal(o, again[0]) and torch.equal(sT, again[1])


# segments of several chunks (of few heads: of one, from three chunks on); lengths that
# end in each of them
@BOTH
@pytest.mark.parametrize("T,B,dk,dv,lengths", [(1537, 1, 64, 64, None), (1600, 1, 40, 72, None),
                                               (1700, 4, 16, 16, [1700, 900, 513, 0]), (2000, 1, 128, 128, None),
                                               (1600, 2, 128, 20, [1600, 64])])
def test_long_sequences_in_segments(T, B, dk, dv, lengths, dtype):
    c = Case(T, B, 1, dk, dv, dtype, lengths=lengths, seed=T + dk)
    # (a training call keeps states besides; one that does not needs its segments' too)
    assert am.gated_delta_workspace_bytes(T, B, 1, dk, dv, dtype=dtype, lengths=None) > 0
    c.check()
    o, sT = c.forward()
    again = c.forward(train=False)
    assert torch.equal(o, again[0]) and torch.equal(sT, again[1])


@BOTH
def test_without_states(dtype):
    Case(70, 3, 2, 24, 24, dtype, seed=4).check(s0=False, dsT=False)
    Case(70, 3, 2, 24, 24, dtype, lengths=[70, 20, 0], seed=5).check(s0=False, dsT=False)
    Case(1600, 1, 1, 24, 24, dtype, seed=6).check(s0=False, dsT=False)


def test_no_frames():
    c = Case(0, 3, 2, 20, 30, torch.float32)
    _, sT = c.forward()
    assert torch.equal(sT, c.s0)
    *_, dlam, ds0 = c.backward()
    assert torch.all(dlam == 0) and torch.equal(ds0, c.dsT)


@BOTH
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (7, 5), (100, 33), (32, 32), (65, 30)])
@pytest.mark.parametrize("lengths", [None, [1, 1, 0, 0]])
def test_one_frame_in_place(dk, dv, lengths, dtype):
    """The form of one frame, the state updated in place, against the oracle and the
    chunked form."""
    c = Case(1, 4, 4, dk, dv, dtype, keys=2, lengths=lengths, seed=dk + dv)
    ref = c.oracle()
    state = c.s0.clone()
    o, _ = c.forward(s0=state, sT=state, train=False)
    assert_close("o", _f64(o), ref[0], BF16_TOL if dtype == torch.bfloat16 else F32_TOL)
    assert_close("sT", _f64(state), ref[1], F32_TOL)
    chunked, sT = c.forward(train=True)
    assert_close("sT, chunked", _f64(sT), ref[1], F32_TOL)
    assert_close("o, chunked", _f64(chunked), ref[0], BF16_TOL if dtype == torch.bfloat16 else F32_TOL)


def test_frames_one_by_one_are_the_sequence():
    c = Case(40, 3, 2, 64, 64, torch.float32, seed=2)
    o, sT = c.forward(train=False)
    state, rows = c.s0.clone(), []
    for t in range(40):
        one = torch.empty((3, 2 * 64), device="cuda")
        am.gated_delta_forward(*[x[3 * t:3 * t + 3] for x in c.cols(c.proj)], c.lam, 1, 3, one, s0=state, sT=state,
                               **c.sizes)
        rows.append(one)
    assert_close("o", _f64(torch.cat(rows)), _f64(o), F32_TOL)
    assert_close("sT", _f64(state), _f64(sT), F32_TOL)


@BOTH
def test_states_and_gradients_in_place(dtype):
    for T in (130, 1600):
        c = Case(T, 2, 1, 40, 24, dtype, seed=T)
        want = c.forward() + c.backward()
        state, grad = c.s0.clone(), c.dsT.clone()
        o, _ = c.forward(s0=state, sT=state)
        got = (o, state) + c.backward(dsT=grad, ds0=grad)
        for w, g in zip(want, got):
            assert torch.equal(w, g)


@BOTH
def test_the_same_bits_each_time_and_nothing_beside(dtype):
    c = Case(150, 3, 4, 40, 24, dtype, keys=2, pad=3, lengths=[150, 70, 3], seed=8)
    first = [t.clone() for t in c.forward() + c.backward()]
    second = c.forward() + c.backward()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    wide = torch.full_like(c.proj, 7.0)
    dlam = torch.empty(4, device="cuda")
    am.gated_delta_backward(*c.cols(c.proj), c.lam, c.T, c.B, c.do, c.ws, *c.cols(wide), dlam, lengths=c.lengths,
                            s0=c.s0, dsT=c.dsT, **c.sizes)
    assert torch.all(wide[:, :3] == 7) and torch.all(wide[:, -3:] == 7)
    outer = torch.full((c.N + 2, c.heads * c.dv + 5), 7.0, dtype=dtype, device="cuda")
    am.gated_delta_forward(*c.cols(c.proj), c.lam, c.T, c.B, outer[1:-1, 2:-3], c.ws, lengths=c.lengths, s0=c.s0,
                           train=True, **c.sizes)
    assert torch.equal(outer[1:-1, 2:-3], first[0])
    assert torch.all(outer[[0, -1]] == 7) and torch.all(outer[:, :2] == 7) and torch.all(outer[:, -3:] == 7)


@BOTH
@pytest.mark.parametrize("what", ["one key", "two keys", "no decay", "all decay", "zero rows", "shut"])
def test_inputs_at_the_edges(what, dtype):
    """Keys that repeat make (I + L)^-1 the difference of neighbours; decays from none to
    all of the state in a frame; rows of zeros have no length; shut gates write nothing."""
    c = Case(130, 2, 2, 32, 32, dtype, seed=3, lam=(2.0, 3.0) if what == "all decay" else (-6.0, -1.0))
    q, k, v, r, b = c.cols(c.proj)
    if what == "one key":
        k.copy_(k[:1].expand_as(k).clone())
        b.fill_(30.0)
        r.fill_(-30.0)
    elif what == "two keys":
        k[::2] = k[:1].clone()
        k[1::2] = k[1:2].clone()
        b.fill_(30.0)
    elif what == "no decay":
        r.fill_(-200.0)
    elif what == "all decay":
        r.fill_(30.0)
    elif what == "zero rows":
        q[5:9], k[3:70], v[60:] = 0, 0, 0
    else:
        b.fill_(-200.0)
    # (where the state's gradient is lost within a frame, or nothing is written, some
    # gradients are differences that cancel to nothing: those are held to the others' size)
    got, ref = c.forward() + c.backward(), c.oracle()
    for name, g, w in zip(("o", "sT", "dq", "dk", "dv", "dr", "db", "dlam", "ds0"), got, ref):
        tol = BF16_TOL if g.dtype == torch.bfloat16 else F32_TOL
        size = max(np.abs(w).max(), 1e-2) + 2.0 ** -20 / tol * c.along.get(name, 0.0)
        if name in ("dr", "dlam"):
            # the gradient of log a is a sum of do o - dv v over the frames of a chunk, each
            # a sum over columns in 32 bits, off by 2^-21 of its terms' magnitudes at most:
            # where the decay has no effect the terms cancel, and that is what is left
            terms = (np.abs(_f64(c.do) * ref[0]) + np.abs(ref[4] * _f64(v))).reshape(130, 2, 2, 32).sum(-1)
            of_log = 2.0 ** -21 * np.stack([terms[:64].sum(0), terms[64:128].sum(0)]).max()
            rate = 8 * np.logaddexp(0, _f64(c.lam)).max()
            size += of_log / tol * (rate / 4 if name == "dr" else 8 * 260)
        assert np.isfinite(_f64(g)).all(), name
        assert np.abs(_f64(g) - w).max() <= tol * size, (name, np.abs(_f64(g) - w).max(), size)


@BOTH
@pytest.mark.parametrize("lam", [1e3, 1e30, 3e38])
def test_decays_to_nothing(lam, dtype):
    """Rates that leave nothing of a state, up to ones past 32 bits: frames alone, and no
    gradient of the gate that shuts (what rounding leaves of it would be multiplied by
    the rate)."""
    c = Case(130, 2, 2, 32, 32, dtype, seed=9, lam=(lam, lam))
    c.cols(c.proj)[3].fill_(3.0)
    got, ref = c.forward() + c.backward(), c.oracle()
    for name, g, w in zip(("o", "sT", "dq", "dk", "dv", "dr", "db", "dlam", "ds0"), got, ref):
        assert np.isfinite(_f64(g)).all(), name
        if name in ("dr", "dlam", "ds0"):
            assert not _f64(g).any() and np.abs(w).max() < 1e-30, name
        else:
            assert_close(name, _f64(g), w, BF16_TOL if g.dtype == torch.bfloat16 else F32_TOL)


def test_another_gpu_is_refused(monkeypatch):
    """(As if the call's stream were the second GPU's.)"""
    c = Case(5, 2, 2, 16, 16, torch.bfloat16, seed=1)
    monkeypatch.setattr(am, "_raw_device", lambda: 1)
    for call in (c.forward, c.backward):
        with pytest.raises(am.AmError, match="GPU"):
            call()


def test_a_nan_stays_in_its_head():
    c = Case(100, 2, 3, 16, 16, torch.float32, seed=1)
    c.cols(c.proj)[2][70, 20] = NAN  # v of head 1, sequence 0, frame 35
    o, sT = c.forward()
    bad = torch.isnan(o.view(100, 2, 3, 16)).any(-1)
    want = torch.zeros_like(bad)
    want[32:, 0, 1] = True  # (frames are summed in blocks of 16)
    assert not (bad & ~want).any() and bad[35:, 0, 1].all()
    assert torch.isnan(sT[0, 1]).any() and torch.isfinite(sT[1]).all() and torch.isfinite(sT[0, [0, 2]]).all()


def test_rows_far_apart():
    """Offsets past 2^32 bytes and 2^31 elements."""
    T, B, stride = 70, 1000, 32768
    big = torch.empty((T * B, stride), dtype=torch.bfloat16, device="cuda")
    c = Case(T, B, 1, 16, 16, seed=2)
    view = big[:, -c.proj.shape[1]:]
    view.copy_(c.proj)
    c.proj, c.s0 = view, c.s0
    o, sT = c.forward()
    rows = torch.arange(B - 3, T * B, B, device="cuda")
    d = Case(T, 1, 1, 16, 16)
    d.proj, d.lam, d.s0 = view[rows].contiguous(), c.lam, c.s0[B - 3:B - 2].contiguous()
    o1, s1 = d.forward()
    assert torch.equal(o[rows], o1) and torch.equal(sT[B - 3], s1[0])


def test_on_another_stream_and_in_a_graph():
    c = Case(130, 3, 2, 64, 64, lengths=[130, 100, 9], seed=5)
    want = [t.clone() for t in c.forward() + c.backward()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.forward() + c.backward()
    side.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w, g)
    o, dproj = torch.empty_like(want[0]), torch.empty_like(c.proj)
    sT, ds0, dlam = torch.empty_like(c.s0), torch.empty_like(c.s0), torch.empty(2, device="cuda")

    def both():
        am.gated_delta_forward(*c.cols(c.proj), c.lam, c.T, c.B, o, c.ws, lengths=c.lengths, s0=c.s0, sT=sT, train=True,
                               **c.sizes)
        am.gated_delta_backward(*c.cols(c.proj), c.lam, c.T, c.B, c.do, c.ws, *c.cols(dproj), dlam, lengths=c.lengths,
                                s0=c.s0, dsT=c.dsT, ds0=ds0, **c.sizes)
    graph = torch.cuda.CUDAGraph()
    both()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        for t in (o, dproj, sT, ds0, dlam):
            t.fill_(NAN)
        if k == 1:  # other values in the same places
            c.proj.copy_(torch.randn_like(c.proj.float()).to(c.proj.dtype))
            want = [t.clone() for t in c.forward() + c.backward()]
            need = am.gated_delta_workspace_bytes(c.T, c.B, 2, 64, 64, lengths=c.lengths, train=True)
            assert c.ws.numel() == need
        graph.replay()
        torch.cuda.synchronize()
        got = (o, sT, *c.cols(dproj), dlam, ds0)
        for w, g in zip(want, got):
            assert torch.equal(w, g)
