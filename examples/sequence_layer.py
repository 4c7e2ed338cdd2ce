"""A recurrent sequence layer trained on what the library simulates, and a
coefficient field fitted to an observed state: the operators as a program uses
them together.

    python examples/sequence_layer.py

`train` simulates Allen-Cahn boxes (adst.forward), records a few probe points
of each over time, and trains a layer to predict each next record:

    n = layer_norm(x W_in);  (a | u) = n W_gate + c;  h = recurrence(a, u)
    y = x + layer_norm(h) W_out

Its gradients come from the operators' VJPs (the states of the recurrence are
recomputed from checkpoints), its parameters from AdamW with 8-bit states and
bfloat16 copies to compute with. It then runs the trained layer one record at
a time on a pool of states (recurrence_step), as a serving program does.

`fit_coefficients` recovers a field K of the variable-coefficient diffusion
from an observed final state: adst.vjp gives dL/dK, AdamW takes the step.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_02197_amd as adst  # noqa: E402

SIGMOID = adst.ADST_GATE_SIGMOID


def probe_records(batch, steps, probes, seed=0, device="cuda"):
    """[batch, steps + 1, probes]: values of an Allen-Cahn box at fixed points, step by step."""
    g = torch.Generator().manual_seed(seed)
    shape = (12, 20, 24)
    at = torch.randperm(shape[0] * shape[1] * shape[2], generator=g)[:probes].to(device)
    out = torch.empty(batch, steps + 1, probes, device=device)
    for b in range(batch):
        x = (torch.rand(shape, generator=g) * 2 - 1).to(device)
        for t in range(steps + 1):
            out[b, t] = x.view(-1)[at]
            x = adst.forward(adst.ADST_ALLENCAHN3D7, x, steps=1)
    return out


class SequenceLayer:
    """The layer of this file's head. dtype: what activations and the weights' copies are in
    (float64: the parameters too)."""

    def __init__(self, probes, width, dtype=torch.bfloat16, bits=8, lr=3e-3, seed=0,
                 device="cuda"):
        g = torch.Generator().manual_seed(seed)
        held = torch.float64 if dtype == torch.float64 else torch.float32

        def matrix(n, m):
            return (torch.randn(n, m, generator=g) / n ** 0.5).to(held).to(device)

        ones, zeros = (torch.full((width,), v, dtype=held, device=device) for v in (1.0, 0.0))
        gate = torch.zeros(2 * width, dtype=held, device=device)
        gate[:width] = torch.linspace(0.0, 4.0, width)  # memories of two to fifty steps
        self.names = ("W_in", "w1", "b1", "W_gate", "c", "w2", "b2", "W_out")
        values = (matrix(probes, width), ones.clone(), zeros.clone(), matrix(width, 2 * width),
                  gate, ones.clone(), zeros.clone(), matrix(width, probes) * 0.1)
        self.width, self.dtype = width, dtype
        self.held = dict(zip(self.names, values))
        copies = None
        if dtype != held:
            copies = [v.to(dtype) for v in values]
        self.use = dict(zip(self.names, copies or values))
        decay = [0.01 if v.dim() == 2 else 0.0 for v in values]
        self.optimizer = adst.AdamW(values, bits=bits if held == torch.float32 else 32,
                                    copies=copies, lr=lr, betas=(0.9, 0.99), weight_decay=decay)

    def forward(self, x, keep=False):
        """y [B, T, probes] and, with keep, what the gradients need."""
        p = self.use
        B, T, P = x.shape
        flat = x.reshape(B * T, P)
        z = flat @ p["W_in"]
        n1 = adst.layer_norm(z, p["w1"], p["b1"])
        gates = torch.addmm(p["c"], n1["y"], p["W_gate"]).view(B, T, 2 * self.width)
        a, u = gates[..., :self.width], gates[..., self.width:]
        r = adst.recurrence(a, u, gate=SIGMOID, want_ck=keep)
        h = r["h"].view(B * T, self.width)
        n2 = adst.layer_norm(h, p["w2"], p["b2"])
        y = (flat + n2["y"] @ p["W_out"]).view(B, T, P)
        return y, (flat, z, n1, a, u, r, h, n2)

    def gradients(self, kept, dy):
        """The parameters' gradients from dL/dy."""
        p = self.use
        flat, z, n1, a, u, r, h, n2 = kept
        d = dy.reshape(flat.shape)
        g = {"W_out": n2["y"].t() @ d}
        b2 = adst.layer_norm_vjp(h, d @ p["W_out"].t(), n2["mean"], n2["rstd"], p["w2"])
        g["w2"], g["b2"] = b2["dw"], b2["db"]
        b = adst.recurrence_vjp(a, u, b2["dx"].view(a.shape), ck=r["ck"], gate=SIGMOID)
        dg = torch.cat([b["da"], b["du"]], 2).view(flat.shape[0], 2 * self.width)
        g["W_gate"], g["c"] = n1["y"].t() @ dg, dg.sum(0)
        b1 = adst.layer_norm_vjp(z, dg @ p["W_gate"].t(), n1["mean"], n1["rstd"], p["w1"])
        g["w1"], g["b1"] = b1["dw"], b1["db"]
        g["W_in"] = flat.t() @ b1["dx"]
        return [g[k].contiguous() for k in self.names]

    def loss_and_gradients(self, records):
        """Mean squared error of each next record's prediction."""
        x, want = records[:, :-1].to(self.dtype), records[:, 1:]
        y, kept = self.forward(x, keep=True)
        off = y.to(self.held["c"].dtype) - want
        return (off * off).mean(), self.gradients(kept, (off * (2.0 / off.numel())).to(self.dtype))

    def train_step(self, records):
        loss, grads = self.loss_and_gradients(records)
        self.optimizer.step(grads)
        return loss

    def one(self, x, pool, slots):
        """The next records' predictions from one record of each sequence, whose states are rows
        `slots` of the pool."""
        p = self.use
        n = adst.layer_norm(x @ p["W_in"], p["w1"], p["b1"])["y"]
        gates = torch.addmm(p["c"], n, p["W_gate"])
        h = adst.recurrence_step(gates[:, :self.width], gates[:, self.width:], pool, slots,
                                 gate=SIGMOID)
        return x + adst.layer_norm(h, p["w2"], p["b2"])["y"] @ p["W_out"]


def train(batch=16, steps=96, probes=24, width=192, updates=60, **kw):
    """The losses of `updates` steps, and the largest difference between the layer's outputs one
    record at a time and at once."""
    records = probe_records(batch, steps, probes)
    layer = SequenceLayer(probes, width, **kw)
    losses = [layer.train_step(records) for _ in range(updates)]
    x = records[:, :-1].to(layer.dtype)
    whole, _ = layer.forward(x)
    pool = torch.zeros(2 * batch, width, dtype=layer.held["c"].dtype, device=x.device)
    slots = torch.randperm(2 * batch, device=x.device)[:batch].to(torch.int32)
    served = torch.stack([layer.one(x[:, t], pool, slots) for t in range(steps)], 1)
    return [float(v) for v in losses], float((served - whole).abs().max()), whole


def fit_coefficients(n=96, steps=40, updates=40, lr=0.03, device="cuda"):
    """Losses of a fit of K, and the distances of the first and the last K from the true one."""
    g = torch.Generator().manual_seed(1)
    kind, loss = adst.ADST_VARDIFF2D9, adst.ADST_LOSS_HALF_SQ_DIFF
    x0 = torch.rand(n, n, generator=g).to(device)
    true = 0.8 + 0.4 * torch.rand(n // 8, n // 8, generator=g).repeat_interleave(8, 0) \
        .repeat_interleave(8, 1).to(device)
    seen = adst.forward(kind, x0, true, steps)
    K = torch.ones_like(x0)
    optimizer = adst.AdamW([K], lr=lr, betas=(0.9, 0.99), weight_decay=0.0)
    first, losses = float((K - true).norm()), []
    for _ in range(updates):
        out = adst.vjp(kind, x0, K, steps, loss, seen, want_dcoeff=True,
                       budget_bytes=6 * x0.nbytes)
        losses.append(float(out["loss"]))
        optimizer.step([out["dK"]])
    return losses, first, float((K - true).norm())


def main():
    losses, off, _ = train()
    print(f"sequence layer: loss {losses[0]:.4f} -> {losses[-1]:.4f}, "
          f"one record at a time within {off:.3g}")
    losses, first, last = fit_coefficients()
    print(f"coefficient field: loss {losses[0]:.4g} -> {losses[-1]:.4g}, "
          f"distance {first:.3f} -> {last:.3f}")


if __name__ == "__main__":
    main()
