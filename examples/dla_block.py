"""Blocks of decayed linear attention on the library: training steps with clipped gradients, then prefill and decoding.

    h_0 = x,  z_0 = norm(h_0);  for every block:  y = W_o attention(W_q z, W_k z, silu(W_v z)),
    h <- h + res_scale * gate * norm(y),  z <- norm(h)

The norm after a block, its gate and residual, and the norm before the next are one call of sdm_block_norm; attention is
sdm_dla_forward (sdm_dla_step for single tokens), the projections are sdm_linear, the gradients their backward calls,
and sdm_grad_clip ends the step.  Only the weights' update is a torch operation.

    python examples/dla_block.py [--steps 20] [--B 2] [--T 200] [--H 8] [--H_k 4] [--d 64] [--blocks 2]
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


def project(x, W, act="none", keep=False):
    """act(x W^T), and what the backward needs of it."""
    shape = sdm.LinearShape.make(x.shape[0], W.shape[0], W.shape[1], act=act)
    out = torch.empty((x.shape[0], W.shape[0]), dtype=torch.bfloat16, device="cuda")
    pre = torch.empty_like(out) if keep else None
    sdm.linear(shape, x, W, out, pre=pre, workspace=bytes_(sdm.linear_workspace_bytes(shape)))
    return out, pre


def project_back(x, W, pre, dout, act="none"):
    shape = sdm.LinearShape.make(x.shape[0], W.shape[0], W.shape[1], act=act)
    dx, dW = torch.empty_like(x), torch.empty_like(W)
    sdm.linear_backward(shape, x, W, pre, dout, dx, dW, None, bytes_(sdm.linear_backward_workspace_bytes(shape)))
    return dx, dW


class Blocks:
    """d_model = H * d; q and k have H_k heads of d, v has H.  The gate is a row for every sequence."""

    def __init__(self, n, H, H_k, d, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.H, self.H_k, self.d, self.dm = n, H, H_k, d, H * d
        rows = dict(q=H_k * d, k=H_k * d, v=H * d, o=self.dm)
        self.W = {}
        for i in range(n):
            for name, r in rows.items():
                self.W[f"{name}{i}"] = (torch.randn((r, self.dm), generator=g, device="cuda") / self.dm ** 0.5).bfloat16()
        self.v = {"pre0": torch.ones(self.dm, device="cuda")}
        for i in range(n):
            self.v[f"post{i}"], self.v[f"scale{i}"] = torch.ones(self.dm, device="cuda"), torch.full((self.dm,), 0.5, device="cuda")
            self.v[f"pre{i + 1}"] = torch.ones(self.dm, device="cuda")
        self.log_decay = -torch.exp2(-1 - 9 * torch.arange(H, device="cuda") / max(1, H - 1)).float()

    def shapes(self, B, T):
        return (sdm.DlaShape.make(B, self.H, T, self.d, self.d, H_k=self.H_k, layout="token_major", scale=1 / self.d),
                sdm.BlockNormShape.make(B * T, self.dm, gate_rows=T))

    def heads(self, x, B, T):
        return x.view(B, T, -1, self.d)

    def forward(self, x, gate, states, B, T, lengths=None, train=False, step=None):
        """x [B * T, d_model], gate [blocks, B, d_model], states: per block [B, H, d, d] float32 (a cache of them with
        `step`, the sequences' rows), updated in place.  Returns the last norm's output and what the backward needs."""
        dla, norm = self.shapes(B, T)
        h, z, kept = x, torch.empty_like(x), []
        sdm.block_norm(norm, x, None, None, z, gamma_pre=self.v["pre0"])
        for i in range(self.n):
            s = {"z": z, "h0": h}
            for name in "qkv":
                s[name], s["pre_" + name] = project(z, self.W[f"{name}{i}"], "silu" if name == "v" else "none", train and name == "v")
            if train:
                s["state0"] = states[i].clone()
            y = torch.empty_like(s["v"])
            q, k, v = (self.heads(s[name], B, T) for name in "qkv")
            if step is None:
                sdm.dla_forward(dla, q, k, v, self.log_decay, states[i], self.heads(y, B, T), bytes_(sdm.dla_workspace_bytes(dla)), lengths=lengths)
            else:
                sdm.dla_step(dla, q, k, v, self.log_decay, states[i], self.heads(y, B, T), slots=step)
            s["y"], (s["out"], _) = y, project(y, self.W[f"o{i}"])
            h, z = torch.empty_like(x), torch.empty_like(x)
            sdm.block_norm(norm, s["h0"], s["out"], h, z, gate=gate[i], res_scale=self.v[f"scale{i}"],
                           gamma_post=self.v[f"post{i}"], gamma_pre=self.v[f"pre{i + 1}"])
            s["h"] = h
            kept.append(s)
        return z, (x, kept)

    def backward(self, kept, gate, dz, B, T, lengths=None):
        """Gradients of the weights (bf16), of the vectors (float32), of the gates and of x for dz = dL/dz."""
        dla, norm = self.shapes(B, T)
        x, kept = kept
        gW, gv, dgate = {}, {}, torch.empty_like(gate)
        ws, dh = bytes_(sdm.block_norm_backward_workspace_bytes(norm)), None
        for i in reversed(range(self.n)):
            s = kept[i]
            dx, dout = torch.empty_like(x), torch.empty_like(x)
            names = dict(res_scale=f"scale{i}", gamma_post=f"post{i}", gamma_pre=f"pre{i + 1}")
            for n in names.values():
                gv[n] = torch.empty_like(self.v[n])
            sdm.block_norm_backward(norm, s["out"], s["h"], dz, dh, dx, dout, gate=gate[i], dgate=dgate[i],
                                    **{a: self.v[n] for a, n in names.items()}, **{"d" + a: gv[n] for a, n in names.items()}, workspace=ws)
            dy, gW[f"o{i}"] = project_back(s["y"], self.W[f"o{i}"], None, dout)
            d = {n: torch.empty_like(s[n]) for n in "qkv"}
            sdm.dla_backward(dla, *(self.heads(s[n], B, T) for n in "qkv"), self.log_decay, s["state0"], self.heads(dy, B, T), None,
                             *(self.heads(d[n], B, T) for n in "qkv"), None, bytes_(sdm.dla_backward_workspace_bytes(dla)), lengths=lengths)
            dz = 0
            for n in "qkv":
                part, gW[f"{n}{i}"] = project_back(s["z"], self.W[f"{n}{i}"], s["pre_" + n], d[n], "silu" if n == "v" else "none")
                dz = dz + part.float()
            dz, dh = dz.bfloat16(), dx
        gv["pre0"], dx = torch.empty_like(self.v["pre0"]), torch.empty_like(x)
        sdm.block_norm_backward(norm, None, x, dz, dh, dx, None, gamma_pre=self.v["pre0"], dgamma_pre=gv["pre0"], workspace=ws)
        return gW, gv, dgate, dx

    def zero_states(self, B):
        return [torch.zeros((B, self.H, self.d, self.d), device="cuda") for _ in range(self.n)]


def train(model, B, T, steps, lr, max_norm=1.0, seed=1):
    """Fits the blocks' output to that of other blocks of the same shape; returns the losses and the gradients' norms."""
    goal = Blocks(model.n, model.H, model.H_k, model.d, seed=99)
    g = torch.Generator(device="cuda").manual_seed(seed)
    master = {n: w.float() for n, w in model.W.items()}
    x = torch.randn((B * T, model.dm), generator=g, device="cuda").bfloat16()
    gate = torch.sigmoid(torch.randn((model.n, B, model.dm), generator=g, device="cuda")).bfloat16()
    want = goal.forward(x, gate, goal.zero_states(B), B, T)[0].float()
    stats, losses, norms = torch.empty(2, device="cuda"), [], []
    for _ in range(steps):
        z, kept = model.forward(x, gate, model.zero_states(B), B, T, train=True)
        diff = z.float() - want
        losses.append(float(diff.square().mean()))
        gW, gv, _, _ = model.backward(kept, gate, diff.bfloat16(), B, T)
        grads = sdm.GradList.make(list(gW.values()) + list(gv.values()))
        sdm.grad_clip(grads, max_norm, stats, bytes_(sdm.grad_workspace_bytes(grads)))       # in place
        norms.append(float(stats[0]))
        for n, d in gW.items():
            master[n] -= lr * d.float()
            model.W[n] = master[n].bfloat16()
        for n, d in gv.items():
            model.v[n] -= lr * d
    return losses, norms


def prefill_and_decode(model, B, T, seed=2):
    """The last tokens one by one through a cache of states, against the whole sequence at once; the largest difference
    relative to the outputs' root mean square."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, T, model.dm), generator=g, device="cuda").bfloat16()
    gate = torch.sigmoid(torch.randn((model.n, B, model.dm), generator=g, device="cuda")).bfloat16()
    whole = model.forward(x.reshape(B * T, -1), gate, model.zero_states(B), B, T)[0].view(B, T, -1)
    head, slots = T - 4, torch.arange(B, 0, -1, dtype=torch.int32, device="cuda")
    cache, states = [torch.zeros((B + 3, *s.shape[1:]), device="cuda") for s in model.zero_states(B)], model.zero_states(B)
    model.forward(x[:, :head].reshape(B * head, -1), gate, states, B, head)
    for c, s in zip(cache, states):
        c[slots.long()] = s
    got = torch.stack([model.forward(x[:, t].contiguous(), gate, cache, B, 1, step=slots)[0] for t in range(head, T)], 1)
    return float((got.float() - whole[:, head:].float()).abs().max() / whole.float().square().mean().sqrt())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for n, v in (("steps", 20), ("B", 2), ("T", 200), ("H", 8), ("H_k", 4), ("d", 64), ("blocks", 2)):
        ap.add_argument("--" + n, type=int, default=v)
    a = ap.parse_args(argv)
    model = Blocks(a.blocks, a.H, a.H_k, a.d)
    losses, norms = train(model, a.B, a.T, a.steps, lr=0.05)
    print("loss %.4f -> %.4f in %d steps, gradient norm %.1f -> %.1f, clipped at 1" % (losses[0], losses[-1], a.steps, norms[0], norms[-1]))
    far = prefill_and_decode(model, a.B, a.T)
    print("decoding against the whole sequence: largest difference %.4f of the outputs' root mean square" % far)
    assert sdm.device_status() == 0
    return losses, norms, far


if __name__ == "__main__":
    main()
