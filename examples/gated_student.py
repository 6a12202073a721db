"""A student of gated linear recurrences in place of the LSTM layers, trained
against sparse teacher targets with AdamW:

    res = x Win^T;  y = norm(res)
    each block:  x, r, i = y Wp^T;  gate = y Wg^T;  h = recurrence(x, r, i)
                 res, y = res + scale norm(h silu(gate)) w_post, norm(res)
    logits = y Wo^T + bo

The recurrence, what stands between two blocks, the loss and the optimizer are
the library's kernels; the projections are plain matrix products.

With --mixer delta a block's memory is a matrix for each 64 channels, the gated delta
rule over q, k, v, r, b = y Wp^T in the recurrence's place.  With --projections 8 the
blocks' products and their gradients are in 8 bits: the norm leaves in 8 bits, Wp and Wg
are quantised again after each step.

    python -m examples.gated_student [--steps 100] [--bits 8] [--dtype f32]
                                     [--mixer delta] [--projections 8]
"""

import argparse

import torch

from paper_1904_10584_amd import binding as am
from paper_1904_10584_amd import synth

F32, BF16 = torch.float32, torch.bfloat16


class GatedStudent:
    """Parameters, gradients and optimizer state of the student, and its calls
    for one batch shape (T frames, B sequences, `lengths` sorted or None)."""

    def __init__(self, layers, input_dim, hidden, classes, T, B, K, lengths=None, dtype=BF16, bits=32,
                 lr=2e-3, weight_decay=0.01, seed=0, mixer="gated", projections=16):
        assert hidden % 64 == 0 or mixer == "gated", "the delta rule's heads have 64 channels"
        assert projections == 16 or dtype == BF16, "products in 8 bits are written in bf16"
        self.delta, self.q8, self.heads = mixer == "delta", projections == 8, hidden // 64
        # columns of a block's projection: x, r, i, or q, k, v and two gates a head
        self.at = [0, hidden, 2 * hidden, 3 * hidden]
        if self.delta:
            self.at += [3 * hidden + self.heads, 3 * hidden + 2 * self.heads]
        self.layers, self.H, self.T, self.B, self.lengths, self.dtype = layers, hidden, T, B, lengths, dtype
        self.N = T * B if lengths is None else int(sum(lengths))
        self.lr, self.steps, N, H = lr, 0, self.N, hidden
        gen = torch.Generator().manual_seed(seed)
        self.master, self.weights, self.grads = {}, {}, {}
        matrix = lambda n, k: (torch.rand((n, k), generator=gen) * 2 - 1) * k ** -0.5  # noqa: E731
        self._add("Win", matrix(H, input_dim), dtype)
        self._add("w0", torch.ones(H))
        for l in range(layers):
            self._add(f"Wp{l}", matrix(self.at[-1], H), dtype)
            self._add(f"Wg{l}", matrix(H, H), dtype)
            # decays of an open gate between 0.9 and 0.999 (c = 8)
            rate = -torch.log(torch.rand(self.heads if self.delta else H, generator=gen) * 0.099 + 0.9) / 8.0
            self._add(f"lam{l}", torch.log(torch.expm1(rate)))
            self._add(f"post{l}", torch.ones(H))
            self._add(f"scale{l}", torch.full((H,), layers ** -0.5))
            self._add(f"next{l}", torch.ones(H))
        self._add("Wo", matrix(classes, H), dtype)
        self._add("bo", torch.zeros(classes), dtype)

        new = lambda shape, kind=dtype: torch.empty(shape, dtype=kind, device="cuda")  # noqa: E731
        self.res = [new((N, H), F32) for _ in range(layers + 1)]
        self.y = [new((N, H)) for _ in range(layers + 1)]
        self.rstd = [new((N, 2), F32) for _ in range(layers + 1)]
        self.h = [new((N, H)) for _ in range(layers)]
        need = (am.gated_delta_workspace_bytes(T, B, self.heads, 64, 64, dtype=dtype, lengths=lengths, train=True)
                if self.delta else am.gated_recurrence_workspace_bytes(T, B, H, lengths, train=True))
        self.rec_ws = [new(max(need, 1), torch.uint8) for _ in range(layers)]
        self.norm_ws = new(am.gated_norm_workspace_bytes(N, H), torch.uint8)
        self.ce_ws = new(am.ce_workspace_bytes(N), torch.uint8)
        self.loss, self.dlogits, self.guard = new(1, F32), new((N, classes)), new(1, F32)
        self.optimizer = self._optimizer(bits, weight_decay)
        self.codes = {}
        if self.q8:
            P, sizes = self.at[-1], am.q8_matmul_workspace_bytes
            self.y8 = am.q8_empty(N, H)
            self.q8_ws = new(max(1, sizes(P, H, N), sizes(H, H, N), sizes(N, P, H), sizes(N, H, P), sizes(N, H, H)), torch.uint8)
            self._quantise_weights()

    def _quantise_weights(self):
        """The blocks' weights in 8 bits, as they lie and transposed."""
        for k, w in self.master.items():
            if k[:2] in ("Wp", "Wg"):
                if k not in self.codes:
                    self.codes[k] = am.q8_empty(*w.shape, True) + am.q8_empty(*w.shape[::-1], True)
                am.q8_quantise(w, *self.codes[k], tiles=True)

    def _in_8_bits(self, x, transposed):
        """x in 8 bits as it lies, or transposed."""
        if transposed:
            out = am.q8_empty(*x.shape[::-1])
            am.q8_quantise(x, codes_t=out[0], scales_t=out[1])
        else:
            out = am.q8_empty(*x.shape)
            am.q8_quantise(x, *out)
        return out

    def _norm(self, l, res, **parts):
        """The norm before block l; in 8 bits too where the block's products are."""
        if self.q8 and l < self.layers:
            am.gated_norm_forward_q8(res, *self.y8, y=self.y[l], rstd=self.rstd[l], **parts)
        else:
            am.gated_norm_forward(res, y=self.y[l], rstd=self.rstd[l], **parts)

    def _project(self, y, y8, name, ws=None):
        """y W^T; y8: y in 8 bits.  A stream's few rows may need more workspace than
        training's many, and may run beside them: without `ws` they have their own."""
        if not self.q8:
            return y @ self.weights[name].t()
        (N, K), n = y.shape, self.master[name].shape[0]
        out = torch.empty((N, n), dtype=BF16, device="cuda")
        if ws is None:
            ws = torch.empty(am.q8_matmul_workspace_bytes(N, n, K), dtype=torch.uint8, device="cuda")
        am.q8_matmul(*y8, *self.codes[name][:2], out, tiles=True, ws=ws)
        return out

    def _project_back(self, y, grads):
        """The gradient of y and of the weights from [(name, dL/d(y W^T))]."""
        g, w = self.grads, self.weights
        if not self.q8:
            dy = None
            for name, d in grads:
                torch.mm(d.t(), y, out=g[name])
                dy = d @ w[name] if dy is None else torch.addmm(dy, d, w[name])
            return dy
        dy, yt = torch.empty_like(y), self._in_8_bits(y, True)
        for n, (name, d) in enumerate(grads):
            am.q8_matmul(*self._in_8_bits(d, True), *yt, g[name], ws=self.q8_ws)
            am.q8_matmul(*self._in_8_bits(d, False), *self.codes[name][2:], dy, tiles=True, accumulate=n > 0,
                         ws=self.q8_ws)
        return dy

    def _mix(self, p, l, o, ws, T, B, lengths, train, s0=None, sT=None):
        """A block's memory over its projection."""
        lam = self.weights[f"lam{l}"]
        if self.delta:
            am.gated_delta_forward(*self._parts(p), lam, T, B, o, ws, heads=self.heads, lengths=lengths, s0=s0, sT=sT,
                                   train=train)
        else:
            am.gated_recurrence_forward(*self._parts(p), lam, T, B, o, ws, lengths=lengths, h0=s0, hT=sT, train=train)

    def _add(self, name, value, kind=F32):
        self.master[name] = value.to("cuda", F32)
        self.weights[name] = self.master[name] if kind == F32 else self.master[name].to(kind)
        self.grads[name] = torch.zeros_like(self.weights[name])

    def _optimizer(self, bits, weight_decay):
        """One list of tensors for each type of gradient."""
        lists = {}
        for k, w in self.master.items():
            t = dict(master=w, grad=self.grads[k], weight_decay=weight_decay if w.dim() == 2 else 0.0)
            if self.weights[k] is not w:
                t["weights_bf16"] = self.weights[k]
            for m in ("m", "v"):
                t[m] = torch.zeros(w.numel(), dtype=F32 if bits == 32 else torch.float8_e4m3fn, device="cuda")
                if bits == 8:
                    t[m + "_scale"] = torch.zeros(am.adamw_scales(w.numel()), device="cuda")
            lists.setdefault(self.grads[k].dtype, []).append(t)
        return [am.AdamWTensors(v) for v in lists.values()]

    def _parts(self, t):
        return [t[:, a:b] for a, b in zip(self.at, self.at[1:])]

    def forward(self, x):
        """Logits [N][C] fp32 of packed frames x; keeps what backward reads."""
        w = self.weights
        self.x = x.to(self.dtype)
        self.p, self.g = [], []
        self.res[0].copy_(self.x @ w["Win"].t())
        self._norm(0, self.res[0], w_next=w["w0"])
        for l in range(self.layers):
            for parts, name in ((self.p, "Wp"), (self.g, "Wg")):
                parts.append(self._project(self.y[l], self.q8 and self.y8, f"{name}{l}", self.q8 and self.q8_ws))
            self._mix(self.p[l], l, self.h[l], self.rec_ws[l], self.T, self.B, self.lengths, True)
            self._norm(l + 1, self.res[l], o=self.h[l], gate=self.g[l], w_post=w[f"post{l}"],
                       scale=w[f"scale{l}"], w_next=w[f"next{l}"], res_out=self.res[l + 1])
        return torch.addmm(w["bo"], self.y[-1], w["Wo"].t()).float()

    def backward(self, dz):
        """Gradients of every parameter from dL/dlogits."""
        w, g = self.weights, self.grads
        torch.mm(dz.t(), self.y[-1], out=g["Wo"])
        torch.sum(dz, 0, out=g["bo"])
        dy, dres = dz @ w["Wo"], None
        for l in reversed(range(self.layers)):
            below, dh, dg = torch.empty_like(self.res[l]), torch.empty_like(self.h[l]), torch.empty_like(self.g[l])
            am.gated_norm_backward(self.res[l], self.rstd[l + 1], below, self.norm_ws, o=self.h[l],
                                   gate=self.g[l], w_post=w[f"post{l}"], scale=w[f"scale{l}"],
                                   w_next=w[f"next{l}"], dy=dy, dres_out=dres, do=dh, dgate=dg,
                                   dw_post=g[f"post{l}"], dscale=g[f"scale{l}"], dw_next=g[f"next{l}"])
            dp, dres = torch.empty_like(self.p[l]), below
            back = am.gated_delta_backward if self.delta else am.gated_recurrence_backward
            back(*self._parts(self.p[l]), w[f"lam{l}"], self.T, self.B, dh, self.rec_ws[l], *self._parts(dp),
                 g[f"lam{l}"], lengths=self.lengths, **(dict(heads=self.heads) if self.delta else {}))
            dy = self._project_back(self.y[l], [(f"Wg{l}", dg), (f"Wp{l}", dp)])
        below = torch.empty_like(self.res[0])
        am.gated_norm_backward(self.res[0], self.rstd[0], below, self.norm_ws, w_next=w["w0"], dy=dy,
                               dres_out=dres, dw_next=g["w0"])
        torch.mm(below.to(self.dtype).t(), self.x, out=g["Win"])

    def step(self, x, idx, prob):
        """One training step; the loss stays on the GPU.  A loss that is not finite
        leaves weights and moments as they were (so does a forward pass that timed
        out: its outputs are NaN)."""
        logits = self.forward(x)
        am.sparse_soft_ce(logits, idx, prob, self.loss, self.dlogits, self.ce_ws)
        self.backward(self.dlogits)
        self.steps += 1
        torch.mul(self.loss, 0.0, out=self.guard).add_(1.0)  # 1, or NaN
        for tensors in self.optimizer:
            am.adamw_apply(tensors, lr=self.lr, step=self.steps, beta2=0.99, seed=self.steps,
                           grad_scale=self.guard)
        if self.q8:
            self._quantise_weights()
        return self.loss

    def check(self):
        """Synchronise; raise if a wait of the last step's recurrences timed out."""
        if self.delta:  # (which has none)
            return torch.cuda.synchronize()
        for ws in self.rec_ws:
            am.workspace_check(ws)

    def stream(self, states, x):
        """Logits of the next frame of each stream (x [B][D]); states [layers][B][H] (of the
        delta rule [layers][B][heads][64][64]) fp32 are carried on in place."""
        w, B = self.weights, x.shape[0]
        res = (x.to(self.dtype) @ w["Win"].t()).float()
        y = torch.empty((B, self.H), dtype=self.dtype, device="cuda")
        h, y8 = torch.empty_like(y), am.q8_empty(B, self.H) if self.q8 else None

        def norm(l, **parts):
            if self.q8 and l < self.layers:
                am.gated_norm_forward_q8(res, *y8, **parts)
            else:
                am.gated_norm_forward(res, y=y, **parts)

        norm(0, w_next=w["w0"])
        for l in range(self.layers):
            p, gate = self._project(y, y8, f"Wp{l}"), self._project(y, y8, f"Wg{l}")
            self._mix(p, l, h, None, 1, B, None, False, states[l], states[l])
            norm(l + 1, o=h, gate=gate, w_post=w[f"post{l}"], scale=w[f"scale{l}"], w_next=w[f"next{l}"], res_out=res)
        return torch.addmm(w["bo"], y, w["Wo"].t()).float()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--bits", type=int, default=32, choices=(32, 8))
    ap.add_argument("--dtype", default="bf16", choices=("bf16", "f32"))
    ap.add_argument("--mixer", default="gated", choices=("gated", "delta"))
    ap.add_argument("--projections", type=int, default=16, choices=(16, 8))
    a = ap.parse_args()
    s = synth.WORKLOADS["tiny-2x64"]
    T, B, K = s["T"], s["B"], s["K"]
    student = GatedStudent(s["layers"], s["input_dim"], s["hidden"], s["classes"], T, B, K,
                           dtype=BF16 if a.dtype == "bf16" else F32, bits=a.bits, mixer=a.mixer,
                           projections=a.projections)
    x = torch.from_numpy(synth.features(T * B, s["input_dim"])).cuda()
    idx, prob = (torch.from_numpy(v).cuda() for v in synth.teacher_targets(T * B, s["classes"], K, s["mass"]))
    for k in range(a.steps):
        loss = student.step(x, idx, prob)
        if k % 10 == 0 or k + 1 == a.steps:
            student.check()
            print(f"step {k}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
