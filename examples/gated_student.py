"""A student of gated linear recurrences in place of the LSTM layers, trained
against sparse teacher targets with AdamW:

    res = x Win^T;  y = norm(res)
    each block:  x, r, i = y Wp^T;  gate = y Wg^T;  h = recurrence(x, r, i)
                 res, y = res + scale norm(h silu(gate)) w_post, norm(res)
    logits = y Wo^T + bo

The recurrence, what stands between two blocks, the loss and the optimizer are
the library's kernels; the projections are plain matrix products.

    python -m examples.gated_student [--steps 100] [--bits 8] [--dtype f32]
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
                 lr=2e-3, weight_decay=0.01, seed=0):
        self.layers, self.H, self.T, self.B, self.lengths, self.dtype = layers, hidden, T, B, lengths, dtype
        self.N = T * B if lengths is None else int(sum(lengths))
        self.lr, self.steps, N, H = lr, 0, self.N, hidden
        gen = torch.Generator().manual_seed(seed)
        self.master, self.weights, self.grads = {}, {}, {}
        matrix = lambda n, k: (torch.rand((n, k), generator=gen) * 2 - 1) * k ** -0.5  # noqa: E731
        self._add("Win", matrix(H, input_dim), dtype)
        self._add("w0", torch.ones(H))
        for l in range(layers):
            self._add(f"Wp{l}", matrix(3 * H, H), dtype)
            self._add(f"Wg{l}", matrix(H, H), dtype)
            # decays of an open gate between 0.9 and 0.999 (c = 8)
            rate = -torch.log(torch.rand(H, generator=gen) * 0.099 + 0.9) / 8.0
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
        need = am.gated_recurrence_workspace_bytes(T, B, H, lengths, train=True)
        self.rec_ws = [new(max(need, 1), torch.uint8) for _ in range(layers)]
        self.norm_ws = new(am.gated_norm_workspace_bytes(N, H), torch.uint8)
        self.ce_ws = new(am.ce_workspace_bytes(N), torch.uint8)
        self.loss, self.dlogits, self.guard = new(1, F32), new((N, classes)), new(1, F32)
        self.optimizer = self._optimizer(bits, weight_decay)

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
        H = self.H
        return t[:, :H], t[:, H:2 * H], t[:, 2 * H:]

    def forward(self, x):
        """Logits [N][C] fp32 of packed frames x; keeps what backward reads."""
        w = self.weights
        self.x = x.to(self.dtype)
        self.p, self.g = [], []
        self.res[0].copy_(self.x @ w["Win"].t())
        am.gated_norm_forward(self.res[0], w_next=w["w0"], y=self.y[0], rstd=self.rstd[0])
        for l in range(self.layers):
            self.p.append(self.y[l] @ w[f"Wp{l}"].t())
            self.g.append(self.y[l] @ w[f"Wg{l}"].t())
            am.gated_recurrence_forward(*self._parts(self.p[l]), w[f"lam{l}"], self.T, self.B, self.h[l],
                                        self.rec_ws[l], lengths=self.lengths, train=True)
            am.gated_norm_forward(self.res[l], o=self.h[l], gate=self.g[l], w_post=w[f"post{l}"],
                                  scale=w[f"scale{l}"], w_next=w[f"next{l}"], res_out=self.res[l + 1],
                                  y=self.y[l + 1], rstd=self.rstd[l + 1])
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
            am.gated_recurrence_backward(*self._parts(self.p[l]), w[f"lam{l}"], self.T, self.B, dh,
                                         self.rec_ws[l], *self._parts(dp), g[f"lam{l}"], lengths=self.lengths)
            torch.mm(dp.t(), self.y[l], out=g[f"Wp{l}"])
            torch.mm(dg.t(), self.y[l], out=g[f"Wg{l}"])
            dy = torch.addmm(dg @ w[f"Wg{l}"], dp, w[f"Wp{l}"])
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
        return self.loss

    def check(self):
        """Synchronise; raise if a wait of the last step's recurrences timed out."""
        for ws in self.rec_ws:
            am.workspace_check(ws)

    def stream(self, states, x):
        """Logits of the next frame of each stream (x [B][D]); states [layers][B][H]
        fp32 are carried on in place."""
        w, B = self.weights, x.shape[0]
        res = (x.to(self.dtype) @ w["Win"].t()).float()
        y = torch.empty((B, self.H), dtype=self.dtype, device="cuda")
        h = torch.empty_like(y)
        am.gated_norm_forward(res, w_next=w["w0"], y=y)
        for l in range(self.layers):
            p, gate = y @ w[f"Wp{l}"].t(), y @ w[f"Wg{l}"].t()
            am.gated_recurrence_forward(*self._parts(p), w[f"lam{l}"], 1, B, h, h0=states[l], hT=states[l])
            am.gated_norm_forward(res, o=h, gate=gate, w_post=w[f"post{l}"], scale=w[f"scale{l}"],
                                  w_next=w[f"next{l}"], res_out=res, y=y)
        return torch.addmm(w["bo"], y, w["Wo"].t()).float()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--bits", type=int, default=32, choices=(32, 8))
    ap.add_argument("--dtype", default="bf16", choices=("bf16", "f32"))
    a = ap.parse_args()
    s = synth.WORKLOADS["tiny-2x64"]
    T, B, K = s["T"], s["B"], s["K"]
    student = GatedStudent(s["layers"], s["input_dim"], s["hidden"], s["classes"], T, B, K,
                           dtype=BF16 if a.dtype == "bf16" else F32, bits=a.bits)
    x = torch.from_numpy(synth.features(T * B, s["input_dim"])).cuda()
    idx, prob = (torch.from_numpy(v).cuda() for v in synth.teacher_targets(T * B, s["classes"], K, s["mass"]))
    for k in range(a.steps):
        loss = student.step(x, idx, prob)
        if k % 10 == 0 or k + 1 == a.steps:
            student.check()
            print(f"step {k}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
