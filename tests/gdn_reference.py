"""The gated delta rule and the linear layer in 64 bits, token by token from the definitions."""
from __future__ import annotations

import math

import torch

F64 = torch.float64


def heads(x, H, token_major):
    """[B, Hk, T, d] or [B, T, Hk, d] -> [B, H, T, d] in 64 bits."""
    x = x.to(F64)
    x = x.transpose(1, 2) if token_major else x
    return x.repeat_interleave(H // x.shape[1], 1)


def gdn(q, k, v, alpha, beta, state, scale, lengths=None, token_major=False):
    """y (in the layout of v) and the last state; differentiable in every floating argument."""
    B, H, T = alpha.shape
    q, k, v = (heads(x, H, token_major) for x in (q, k, v))
    al, be, S = alpha.to(F64), beta.to(F64), state.to(F64)
    ends = torch.full((B,), T, device=S.device) if lengths is None else lengths.to(S.device).long()
    ys = []
    for t in range(T):
        on = (t < ends)[:, None, None]
        zero = torch.zeros((), dtype=F64, device=S.device)
        kt, qt, vt = (torch.where(on, x[:, :, t], zero) for x in (k, q, v))
        a, b = torch.where(on[..., 0], al[:, :, t], zero + 1), torch.where(on[..., 0], be[:, :, t], zero)
        Sd = a[..., None, None] * S
        e = vt - torch.einsum("bhkv,bhk->bhv", Sd, kt)
        S = Sd + b[..., None, None] * kt[..., None] * e[..., None, :]
        ys.append(torch.where(on, scale * torch.einsum("bhkv,bhk->bhv", S, qt), zero))
    y = torch.stack(ys, 2) if ys else v[:, :, :0]
    return (y.transpose(1, 2) if token_major else y), S


def gdn_grads(q, k, v, alpha, beta, state, scale, dy, dstate, lengths=None, token_major=False):
    """Gradients of sum <dy, y> + <dstate, S_T> by reverse-mode differentiation of gdn in 64 bits."""
    live = [x.to(F64).clone() for x in (q, k, v, alpha, beta, state)]
    if lengths is not None:                      # what padded places hold has no gradient and no value
        B, _, T = alpha.shape
        pad = torch.arange(T, device=alpha.device)[None, :] >= lengths.to(alpha.device)[:, None]
        for i in range(3):
            live[i] = torch.where((pad[:, :, None, None] if token_major else pad[:, None, :, None]), torch.zeros_like(live[i]), live[i])
        for i in (3, 4):
            live[i] = torch.where(pad[:, None, :], torch.zeros_like(live[i]), live[i])
        dy = torch.where((pad[:, :, None, None] if token_major else pad[:, None, :, None]), torch.zeros_like(dy), dy)
    live = [x.requires_grad_(True) for x in live]
    y, S = gdn(*live, scale, lengths, token_major)
    loss = (y * dy.to(F64)).sum() + (S * dstate.to(F64)).sum()
    return torch.autograd.grad(loss, live)


def act(z, name):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))}[name]()


def slope(z, name):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).to(z.dtype), "silu": lambda: s * (1 + z * (1 - s)),
            "gelu": lambda: 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


def rel(got, ref):
    """2-norm of the difference over the 2-norm of the reference (0 where both are zero)."""
    got, ref = got.to(F64), ref.to(F64)
    if not torch.isfinite(got).all():
        return math.inf
    d, n = float((got - ref).norm()), float(ref.norm())
    return d / n if n else (0.0 if d == 0 else math.inf)
