"""A selective state-space layer trained to predict the next token of what the
library simulates, and run one token at a time: the token operators as a program
uses them together.

    python examples/token_layer.py

A token is the bin of a probe point's value in a simulated Allen-Cahn box
(examples/sequence_layer.py), a sequence one probe's bins over time. With e the
tokens' embeddings:

    (x | z) = layer_norm(e) W_in;  c = causal_conv(x);  (delta | B | C) = c W_scan
    h = e + selective_scan(c, delta, A, B, C, z) W_out;  loss = cross entropy of h W_head^T

The gradients come from the operators' VJPs (the scan's states recomputed from
checkpoints, the logits from the saved lse), the parameters from AdamW: matrices
with 8-bit states and bfloat16 copies to compute with, what belongs to a channel
in float32. `serve` then runs the layer a token at a time on pools of windows and
states.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_02197_amd as adst  # noqa: E402
from sequence_layer import probe_records  # noqa: E402

SILU = adst.ADST_ACT_SILU


def probe_tokens(boxes, steps, probes, words, device="cuda"):
    """[boxes * probes, steps + 1] int32: the probes' values in `words` equal bins of [-1, 1]."""
    records = probe_records(boxes, steps, probes, device=device)
    bins = ((records.clamp(-1, 1) + 1) * (0.5 * words)).to(torch.int32).clamp(max=words - 1)
    return bins.transpose(1, 2).reshape(boxes * probes, steps + 1).contiguous()


class TokenLayer:
    """The layer of this file's head. dtype: what activations and the matrices' copies are in
    (float64: all parameters too)."""

    def __init__(self, words, width, states=16, taps=4, dtype=torch.bfloat16, bits=8, lr=3e-3,
                 seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        held = torch.float64 if dtype == torch.float64 else torch.float32

        def matrix(n, m, scale=1.0):
            return (torch.randn(n, m, generator=g) * scale).to(held).to(device)

        def channel(v):
            return v.to(held).to(device)

        by = width ** -0.5
        self.matrices = {"embed": matrix(words, width), "W_in": matrix(width, 2 * width, by),
                         "W_scan": matrix(width, width + 2 * states, by),
                         "W_out": matrix(width, width, by), "W_head": matrix(words, width, by)}
        self.channels = {
            "w1": channel(torch.ones(width)), "b1": channel(torch.zeros(width)),
            "conv": matrix(taps, width, taps ** -0.5), "conv_b": channel(torch.zeros(width)),
            "log_A": channel(torch.arange(1, states + 1).log().repeat(width, 1)),
            "D": channel(torch.ones(width)),
            "delta_b": channel(torch.linspace(-4.0, 0.0, width))}  # steps of 0.02 to 0.7
        self.width, self.states, self.dtype = width, states, dtype
        copies = None
        if dtype != held:
            copies = [v.to(dtype) for v in self.matrices.values()]
        self.use = {**dict(zip(self.matrices, copies or self.matrices.values())), **self.channels}
        opt = dict(lr=lr, betas=(0.9, 0.99))
        self.optimizers = (
            adst.AdamW(list(self.matrices.values()), copies=copies, weight_decay=0.01,
                       bits=bits if held == torch.float32 else 32, **opt),
            adst.AdamW(list(self.channels.values()), weight_decay=0.0, **opt))

    def _scan_inputs(self, c):
        """delta, B and C, which are parts of one product's rows."""
        p = c.reshape(-1, self.width) @ self.use["W_scan"]
        p = p.view(*c.shape[:-1], self.width + 2 * self.states)
        return p.split([self.width, self.states, self.states], -1)

    def forward(self, tokens, lens=None, keep=False):
        """h [B, T, width] and what the gradients need."""
        p = self.use
        B, T = tokens.shape
        e = p["embed"][tokens.long()].view(B * T, self.width)
        n = adst.layer_norm(e, p["w1"], p["b1"])
        xz = (n["y"] @ p["W_in"]).view(B, T, 2 * self.width)
        x, z = xz[..., :self.width], xz[..., self.width:]
        c = adst.causal_conv(x, p["conv"], p["conv_b"], lens=lens, act=SILU)["y"]
        delta, Bm, Cm = self._scan_inputs(c)
        A = -p["log_A"].exp()
        s = adst.selective_scan(c, delta, A, Bm, Cm, D=p["D"], z=z, delta_bias=p["delta_b"],
                                lens=lens, softplus=True, want_ck=keep)
        h = e + s["y"].view(B * T, self.width) @ p["W_out"]
        return h, (e, n, x, z, c, delta, Bm, Cm, A, s)

    def loss_and_gradients(self, tokens, lens=None):
        """The mean cross entropy of each next token of rows [B, T + 1] (of lens[b] + 1 tokens),
        and the parameters' gradients."""
        p = self.use
        given, want = tokens[:, :-1], tokens[:, 1:].clone()
        B, T = given.shape
        if lens is not None:
            want[torch.arange(T, device=want.device)[None] >= lens[:, None]] = -1
        labels = want.reshape(-1)
        h, (e, n, x, z, c, delta, Bm, Cm, A, s) = self.forward(given, lens, keep=True)
        f = adst.linear_cross_entropy(h, p["W_head"], labels)
        scale = (labels >= 0) / (labels >= 0).sum().clamp(min=1)
        scale = scale.to(f["loss"].dtype)

        g = {}
        r = adst.linear_cross_entropy_vjp(h, p["W_head"], labels, f["lse"], scale)
        dh, g["W_head"] = r["dx"], r["dw"]
        g["W_out"] = s["y"].view(B * T, self.width).t() @ dh
        dy = (dh @ p["W_out"].t()).view(B, T, self.width)
        r = adst.selective_scan_vjp(c, delta, A, Bm, Cm, dy, D=p["D"], z=z,
                                    delta_bias=p["delta_b"], lens=lens, ck=s["ck"], softplus=True)
        g["log_A"], g["D"], g["delta_b"] = r["dA"] * A, r["dD"], r["ddelta_bias"]
        dp = torch.cat([r["ddelta"], r["dB"], r["dC"]], 2).view(B * T, -1)
        g["W_scan"] = c.view(B * T, self.width).t() @ dp
        dc = r["dx"] + (dp @ p["W_scan"].t()).view(B, T, self.width)
        dz = r["dz"]
        r = adst.causal_conv_vjp(x, dc, p["conv"], p["conv_b"], lens=lens, act=SILU)
        g["conv"], g["conv_b"] = r["dw"], r["db"]
        dxz = torch.cat([r["dx"], dz], 2).view(B * T, 2 * self.width)
        g["W_in"] = n["y"].t() @ dxz
        r = adst.layer_norm_vjp(e, dxz @ p["W_in"].t(), n["mean"], n["rstd"], p["w1"])
        g["w1"], g["b1"] = r["dw"], r["db"]
        de = (dh + r["dx"]).to(A.dtype)
        g["embed"] = torch.zeros_like(self.matrices["embed"]).index_add_(
            0, given.reshape(-1).long(), de).to(self.dtype)
        return (f["loss"] * scale).sum(), g

    def train_step(self, tokens, lens=None):
        loss, g = self.loss_and_gradients(tokens, lens)
        for optimizer, names in zip(self.optimizers, (self.matrices, self.channels)):
            optimizer.step([g[k].contiguous() for k in names])
        return loss

    def pools(self, rows):
        """Windows and states of `rows` sequences."""
        device = self.channels["D"].device
        taps = self.channels["conv"].shape[0]
        return (torch.zeros(rows, taps - 1, self.width, dtype=self.dtype, device=device),
                torch.zeros(rows, self.width, self.states, dtype=self.channels["D"].dtype,
                            device=device))

    def one(self, token, pools, slots):
        """h [B, width] after one token [B] of each sequence, whose windows and states are rows
        `slots` of the pools."""
        p = self.use
        e = p["embed"][token.long()]
        xz = adst.layer_norm(e, p["w1"], p["b1"])["y"] @ p["W_in"]
        x, z = xz[:, :self.width], xz[:, self.width:]
        c = adst.causal_conv_step(x, p["conv"], pools[0], p["conv_b"], slots, act=SILU)
        delta, Bm, Cm = self._scan_inputs(c)
        y = adst.selective_scan_step(c, delta, -p["log_A"].exp(), Bm, Cm, pools[1], D=p["D"], z=z,
                                     delta_bias=p["delta_b"], slots=slots, softplus=True)
        return e + y @ p["W_out"]


def serve(layer, tokens):
    """h [B, T, width], a token at a time."""
    B, T = tokens.shape
    pools = layer.pools(2 * B)
    slots = torch.randperm(2 * B, device=tokens.device)[:B].to(torch.int32)
    return torch.stack([layer.one(tokens[:, t], pools, slots) for t in range(T)], 1)


def train(boxes=8, steps=96, probes=8, words=64, width=128, updates=40, **kw):
    """The losses of `updates` steps, and the largest difference between h one token at a time
    and at once."""
    tokens = probe_tokens(boxes, steps, probes, words)
    layer = TokenLayer(words, width, **kw)
    losses = [layer.train_step(tokens) for _ in range(updates)]
    whole = layer.forward(tokens[:, :-1])[0].view(tokens.shape[0], steps, width)
    return [float(v) for v in losses], float((serve(layer, tokens[:, :-1]) - whole).abs().max())


def main():
    losses, off = train()
    print(f"token layer: loss {losses[0]:.4f} -> {losses[-1]:.4f}, "
          f"one token at a time within {off:.3g}")


if __name__ == "__main__":
    main()
