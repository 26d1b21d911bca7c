"""A gated delta rule layer on the library: training steps, then prefill and decoding.

    o = x + W_o y,   y = gated delta rule of q = |silu(W_q x)|, k = |silu(W_k x)| (unit length per head),
    v = silu(W_v x) and the gates alpha, beta of x

runs as sdm_linear (projections with their activation, the output projection with the residual in its
epilogue), sdm_gates, sdm_gdn_forward and, for training, sdm_gdn_backward and sdm_linear_backward; single
tokens go through sdm_gdn_step on a cache of states.  Only the unit lengths of q and k and their gradient
are torch operations.  The gates' own parameters are kept fixed.

    python examples/gdn_layer.py [--steps 20] [--B 2] [--T 200] [--H 16] [--H_k 8] [--d 64]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_07386_gb300 as sdm  # noqa: E402


def bytes_(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


class GatedDeltaLayer:
    """d_model = H * d; q and k have H_k heads of d, v has H."""

    def __init__(self, H, H_k, d, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.H, self.H_k, self.d, self.dm = H, H_k, d, H * d
        rows = dict(q=H_k * d, k=H_k * d, v=H * d, o=self.dm)
        self.W = {n: (torch.randn((r, self.dm), generator=g, device="cuda") / self.dm ** 0.5).bfloat16() for n, r in rows.items()}
        self.gate = [torch.randn((H, self.dm), generator=g, device="cuda").bfloat16() / self.dm ** 0.5 for _ in range(2)]
        self.b_dt = torch.full((H,), -4.0, device="cuda")
        self.A = torch.rand((H,), generator=g, device="cuda") * 4 + 0.5

    def _project(self, x, name, act, pre, residual=None):
        M, W = x.shape[0], self.W[name]
        shape = sdm.LinearShape.make(M, W.shape[0], W.shape[1], act=act)
        out = torch.empty((M, W.shape[0]), dtype=torch.bfloat16, device="cuda")
        kept = torch.empty_like(out) if pre else None
        sdm.linear(shape, x, W, out, residual=residual, pre=kept, workspace=bytes_(sdm.linear_workspace_bytes(shape)))
        return out, kept

    def _inputs(self, x, B, T, train):
        """Projections and gates of x [B * T, d_model]; what the backward needs of them is kept."""
        kept = {"x": x}
        u, heads = {}, {}
        for n in ("q", "k", "v"):
            u[n], kept["pre_" + n] = self._project(x, n, "silu", train)
            h = u[n].view(B, T, -1, self.d)
            if n != "v":
                f = h.float()
                kept["norm_" + n] = f.norm(dim=-1, keepdim=True).clamp(min=1e-6)
                h = (f / kept["norm_" + n]).bfloat16()
            heads[n] = h
        ab = [torch.empty((B, self.H, T), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        sdm.gates(sdm.SdmShape.make(B, self.H, T, self.d, self.d, 64, 1, 1), self.dm, x, *self.gate, self.b_dt, self.A, *ab)
        kept.update(heads, alpha=ab[0], beta=ab[1])
        return kept

    def shape(self, B, T):
        return sdm.GdnShape.make(B, self.H, T, self.d, self.d, H_k=self.H_k, layout="token_major", scale=self.d ** -0.5)

    def forward(self, x, B, T, state, lengths=None, train=False):
        """x [B * T, d_model] -> o; state [B, H, d, d] float32 is updated in place."""
        s = self._inputs(x, B, T, train)
        if train:
            s["state0"] = state.clone()
        y = torch.empty_like(s["v"])
        shape = self.shape(B, T)
        sdm.gdn_forward(shape, s["q"], s["k"], s["v"], s["alpha"], s["beta"], state, y,
                        bytes_(sdm.gdn_workspace_bytes(shape)), lengths=lengths)
        s["y"] = y.view(B * T, self.dm)
        out, _ = self._project(s["y"], "o", "none", False, residual=x)
        return out, s

    def backward(self, s, do, B, T, lengths=None):
        """Gradients of the weights and of x for do = dL/do."""
        grads, dx = {}, do.float()

        def linear_back(name, x, pre, dout, act):
            W = self.W[name]
            shape = sdm.LinearShape.make(x.shape[0], W.shape[0], W.shape[1], act=act)
            d, grads[name] = torch.empty_like(x), torch.empty_like(W)
            sdm.linear_backward(shape, x, W, pre, dout, d, grads[name], None,
                                bytes_(sdm.linear_backward_workspace_bytes(shape)))
            return d

        dy = linear_back("o", s["y"], None, do, "none")
        g = {n: torch.empty_like(s[n]) for n in ("q", "k", "v", "alpha", "beta")}
        shape = self.shape(B, T)
        sdm.gdn_backward(shape, s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["state0"], dy.view(s["v"].shape), None,
                         g["q"], g["k"], g["v"], g["alpha"], g["beta"], None,
                         bytes_(sdm.gdn_backward_workspace_bytes(shape)), lengths=lengths)
        for n in ("q", "k", "v"):
            d = g[n].float()
            if n != "v":                        # through the unit length: what is along q (or k) does not count
                h = s[n].float()
                d = (d - h * (h * d).sum(-1, keepdim=True)) / s["norm_" + n]
            d = d.bfloat16().view(B * T, -1)
            dx = dx + linear_back(n, s["x"], s["pre_" + n], d, "silu").float()
        return grads, dx

    def step(self, x, cache, slots):
        """One token of each sequence: x [B, d_model], cache [n, H, d, d] float32, slots [B] int32."""
        B = x.shape[0]
        s = self._inputs(x, B, 1, False)
        y = torch.empty_like(s["v"])
        sdm.gdn_step(self.shape(B, 1), s["q"], s["k"], s["v"], s["alpha"], s["beta"], cache, y, slots=slots)
        return self._project(y.view(B, self.dm), "o", "none", False, residual=x)[0]


def train(layer, B, T, steps, lr, seed=1):
    """Fits the layer's output to that of another layer of the same shape; returns the losses."""
    goal = GatedDeltaLayer(layer.H, layer.H_k, layer.d, seed=99)
    goal.gate, goal.A = layer.gate, layer.A
    g = torch.Generator(device="cuda").manual_seed(seed)
    master = {n: w.float() for n, w in layer.W.items()}
    x = torch.randn((B * T, layer.dm), generator=g, device="cuda").bfloat16()
    zero = torch.zeros((B, layer.H, layer.d, layer.d), device="cuda")
    want = goal.forward(x, B, T, zero.clone())[0].float()
    losses = []
    for _ in range(steps):
        out, kept = layer.forward(x, B, T, zero.clone(), train=True)
        diff = out.float() - want
        losses.append(float(diff.square().mean()))
        grads, _ = layer.backward(kept, diff.bfloat16(), B, T)
        for n, d in grads.items():
            master[n] -= lr * d.float() / d.float().norm() * master[n].norm()
            layer.W[n] = master[n].bfloat16()
    return losses


def prefill_and_decode(layer, B, T, seed=2):
    """The last tokens one by one through the cache, against the whole sequence at once; the largest
    difference relative to the outputs' root mean square."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, T, layer.dm), generator=g, device="cuda").bfloat16()
    zero = torch.zeros((B, layer.H, layer.d, layer.d), device="cuda")
    whole = layer.forward(x.reshape(B * T, -1), B, T, zero.clone())[0].view(B, T, -1)
    head = T - 4
    cache = torch.zeros((B + 3, layer.H, layer.d, layer.d), device="cuda")
    slots = torch.arange(B, 0, -1, dtype=torch.int32, device="cuda")
    state = zero.clone()
    layer.forward(x[:, :head].reshape(B * head, -1), B, head, state)
    cache[slots.long()] = state
    got = torch.stack([layer.step(x[:, t].contiguous(), cache, slots) for t in range(head, T)], 1)
    diff = (got.float() - whole[:, head:].float()).abs().max()
    return float(diff / whole.float().square().mean().sqrt())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for n, v in (("steps", 20), ("B", 2), ("T", 200), ("H", 16), ("H_k", 8), ("d", 64)):
        ap.add_argument("--" + n, type=int, default=v)
    a = ap.parse_args(argv)
    layer = GatedDeltaLayer(a.H, a.H_k, a.d)
    losses = train(layer, a.B, a.T, a.steps, lr=0.02)
    print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], a.steps))
    far = prefill_and_decode(layer, a.B, a.T)
    print("decoding against the whole sequence: largest difference %.4f of the outputs' root mean square" % far)
    assert sdm.device_status() == 0
    return losses, far


if __name__ == "__main__":
    main()
