"""Decayed linear attention, the block norm and clipping in 64 bits, from the definitions, and how far off is too far."""
from __future__ import annotations

import torch

F64 = torch.float64


def heads(x, H, token_major):
    """[B, Hk, T, d] or [B, T, Hk, d] -> [B, H, T, d] in 64 bits."""
    x = x.to(F64)
    x = x.transpose(1, 2) if token_major else x
    return x.repeat_interleave(H // x.shape[1], 1)


def dla(q, k, v, log_decay, state, scale, lengths=None, token_major=False):
    """y (in the layout of v) and the last state, token by token; differentiable in every floating argument."""
    H = log_decay.shape[0]
    q, k, v = (heads(x, H, token_major) for x in (q, k, v))
    lam, S = torch.exp(log_decay.to(F64))[None, :, None, None], state.to(F64)
    B, _, T, _ = v.shape
    ends = torch.full((B,), T, device=S.device) if lengths is None else lengths.to(S.device).long()
    zero = torch.zeros((), dtype=F64, device=S.device)
    ys = []
    for t in range(T):
        on = (t < ends)[:, None, None]
        kt, qt, vt = (torch.where(on, x[:, :, t], zero) for x in (k, q, v))
        S = torch.where(on[..., None], lam * S + kt[..., None] * vt[..., None, :], S)
        ys.append(torch.where(on, scale * torch.einsum("bhkv,bhk->bhv", S, qt), zero))
    y = torch.stack(ys, 2) if ys else v[:, :, :0]
    return (y.transpose(1, 2) if token_major else y), S


def dla_grads(q, k, v, log_decay, state, scale, dy, dstate, lengths=None, token_major=False):
    """Gradients of sum <dy, y> + <dstate, S_T> by reverse-mode differentiation of dla in 64 bits."""
    live = [x.to(F64).clone().requires_grad_(True) for x in (q, k, v, state)]
    y, S = dla(live[0], live[1], live[2], log_decay, live[3], scale, lengths, token_major)
    loss = (dy.to(F64) * y).sum() + (0 if dstate is None else (dstate.to(F64) * S).sum())
    got = torch.autograd.grad(loss, live, allow_unused=True)
    return [torch.zeros_like(x) if g is None else g for g, x in zip(got, live)]


def rms_norm(x, gamma, eps):
    return gamma * x / (x.square().mean(-1, keepdim=True) + eps).sqrt()


def block_norm(x, y, gate, res_scale, gamma_post, gamma_pre, gate_rows, eps, stored=None):
    """h and z in 64 bits; z is the norm of `stored` (h rounded) where it is given."""
    x = x.to(F64)
    if y is not None:
        u = y.to(F64) if gamma_post is None else rms_norm(y.to(F64), gamma_post.to(F64), eps)
        if gate is not None:
            u = u * gate.to(F64)[torch.arange(x.shape[0], device=x.device) // gate_rows]
        if res_scale is not None:
            u = u * res_scale.to(F64)
        x = x + u
    z = None if gamma_pre is None else rms_norm(x if stored is None else stored.to(F64), gamma_pre.to(F64), eps)
    return x, z


# A value rounded to bf16 is off by at most half a step, 2^-8 of it; float32 results are sums of float32 products, each
# off by 2^-24 of itself or less, of a few hundred terms of either sign: 1e-5 of the result in the 2-norm leaves room for
# results that are smaller than their terms by a factor of ten.  A rounded result adds both.
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
SUMS = 1e-5


def near(got, want, name=""):
    """Values below 2^-126 have no float32 (nor bf16) of full precision and may come out as zero: exp(-200), the decay of a
    head that forgets at once, is 1e-87.  So each value may also be off by 2^-126."""
    limit = HALF[got.dtype] + SUMS
    want = want.to(F64)
    far, size = float((got.to(F64) - want).norm()), float(want.norm())
    assert far <= limit * size + 2.0 ** -126 * want.numel() ** 0.5, (name, far / max(size, 2.0 ** -126), limit)
