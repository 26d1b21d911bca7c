"""The example blocks: attention, norms, projections and clipping in one run, captured and replayed too, its gradients
against differences, and decoding against the whole sequence."""
import importlib.util
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("dla_block_example", os.path.join(ROOT, "examples", "dla_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,H,H_k,d,blocks", [(2, 130, 8, 4, 64, 2), (1, 70, 4, 4, 128, 1)])
def test_runs(example, B, T, H, H_k, d, blocks):
    """Decoding differs by roundings of bf16 activations (2^-8 of values a few times their root mean square, through a
    block's four products and two norms each)."""
    losses, norms, far = example.main(["--steps", "3", "--B", str(B), "--T", str(T), "--H", str(H), "--H_k", str(H_k), "--d", str(d),
                                       "--blocks", str(blocks)])
    assert all(math.isfinite(x) for x in losses + norms) and far < 0.1


def _model64(model, W, v, x, gate, B, T):
    """The example's blocks in 64 bits, differentiable in W, v and gate."""
    import torch
    from dla_reference import dla, rms_norm
    h = x.double()
    z = rms_norm(h, v["pre0"], 1e-6)
    for i in range(model.n):
        q, k = ((z @ W[f"{n}{i}"].mT).view(B, T, -1, model.d) for n in "qk")
        u = torch.nn.functional.silu(z @ W[f"v{i}"].mT).view(B, T, -1, model.d)
        y, _ = dla(q, k, u, model.log_decay, torch.zeros((B, model.H, model.d, model.d), device="cuda"), 1 / model.d, None, True)
        out = rms_norm(y.reshape(B * T, -1) @ W[f"o{i}"].mT, v[f"post{i}"], 1e-6)
        h = h + v[f"scale{i}"] * gate[i].repeat_interleave(T, 0) * out
        z = rms_norm(h, v[f"pre{i + 1}"], 1e-6)
    return z


@pytest.mark.gpu
def test_gradients(example):
    """Against 64 bits, and steps along them change the loss as they change it in 64 bits.  A gradient passes through some 20
    roundings to bf16 (2^-8 / sqrt(3) of a value in the root mean square: 1% in all), and what a norm takes away of it is
    not taken away of the roundings: 5%."""
    import torch
    B, T = 2, 96
    model = example.Blocks(2, 4, 2, 64, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((B * T, model.dm), generator=g, device="cuda").bfloat16()
    gate = torch.sigmoid(torch.randn((model.n, B, model.dm), generator=g, device="cuda")).bfloat16()
    want = torch.randn((B * T, model.dm), generator=g, device="cuda")

    def loss():
        z, kept = model.forward(x, gate, model.zero_states(B), B, T, train=True)
        diff = z.double() - want.double()
        return float(0.5 * diff.square().sum()), kept, diff

    def loss64(W, v):
        return 0.5 * (_model64(model, W, v, x, gate64, B, T) - want.double()).square().sum()

    _, kept, diff = loss()
    gW, gv, dgate, _ = model.backward(kept, gate, diff.bfloat16(), B, T)
    W64, v64 = ({n: w.double().requires_grad_(True) for n, w in d.items()} for d in (model.W, model.v))
    gate64 = gate.double().requires_grad_(True)
    live = list(W64.values()) + list(v64.values()) + [gate64]
    exact = torch.autograd.grad(loss64(W64, v64), live)
    for n, a, e in zip(list(W64) + list(v64) + ["gate"], [gW[n] for n in W64] + [gv[n] for n in v64] + [dgate], exact):
        assert float((a.double() - e).norm()) <= 0.05 * float(e.norm()), n
    for n in ("q0", "v1", "o0"):
        w, d = model.W[n], gW[n].float()
        step, changes = 2e-2 * w.float().norm() / d.norm(), [0.0, 0.0]
        for sign in (1, -1):
            model.W[n] = (w.float() + sign * step * d).bfloat16()
            changes[0] += sign * loss()[0]
            with torch.no_grad():
                changes[1] += sign * float(loss64({**W64, n: model.W[n].double()}, v64))
        model.W[n] = w
        assert abs(changes[0] - changes[1]) <= 0.05 * abs(changes[1]), n


@pytest.mark.gpu
def test_captured_training_step(example):
    """Forward, backward and clipping of two blocks captured once and replayed on new inputs give what eager calls give."""
    import torch
    sdm = example.sdm
    B, T = 2, 150
    model = example.Blocks(2, 4, 2, 64, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((B * T, model.dm), generator=g, device="cuda").bfloat16()
    gate = torch.sigmoid(torch.randn((model.n, B, model.dm), generator=g, device="cuda")).bfloat16()
    dz = torch.randn((B * T, model.dm), generator=g, device="cuda").bfloat16()
    lengths = torch.tensor([T, 61], dtype=torch.int32, device="cuda")
    stats = torch.zeros(2, device="cuda")

    def step():
        z, kept = model.forward(x, gate, model.zero_states(B), B, T, lengths=lengths, train=True)
        gW, gv, dgate, dx = model.backward(kept, gate, dz, B, T, lengths=lengths)
        grads = sdm.GradList.make(list(gW.values()) + list(gv.values()))
        sdm.grad_clip(grads, 0.5, stats, example.bytes_(sdm.grad_workspace_bytes(grads)))
        return [z, dgate, dx] + list(gW.values()) + list(gv.values())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    x.copy_(torch.randn((B * T, model.dm), generator=g, device="cuda"))
    lengths.copy_(torch.tensor([77, T], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    replayed, seen = [o.clone() for o in out], stats.clone()
    assert all(torch.equal(a, b) for a, b in zip(replayed, step())) and torch.equal(seen, stats)
    assert abs(float(torch.sqrt(sum(o.double().square().sum() for o in replayed[3:]))) - 0.5) <= 2e-3 * 0.5
