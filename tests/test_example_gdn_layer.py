"""The example layer: training lowers its loss, decoding agrees with the whole sequence, and its gradients are
those of differences."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("gdn_layer_example", os.path.join(ROOT, "examples", "gdn_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,H,H_k,d", [(2, 130, 16, 8, 64), (1, 70, 4, 4, 128)])
def test_trains_and_decodes(example, B, T, H, H_k, d):
    """Decoding differs by roundings of bf16 activations (2^-8 of values a few times their root mean square)."""
    losses, far = example.main(["--steps", "12", "--B", str(B), "--T", str(T), "--H", str(H), "--H_k", str(H_k), "--d", str(d)])
    assert losses[-1] < 0.8 * losses[0]
    assert far < 0.1


@pytest.mark.gpu
def test_weight_gradients_point_downhill(example):
    """A step of length 1e-2 of a weight's norm along its gradient changes the loss by the gradient's norm
    times the step, within 15% (bf16 weights and activations)."""
    import torch
    B, T = 2, 96
    layer = example.GatedDeltaLayer(8, 4, 64, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((B * T, layer.dm), generator=g, device="cuda").bfloat16()
    want = torch.randn((B * T, layer.dm), generator=g, device="cuda")
    zero = torch.zeros((B, layer.H, layer.d, layer.d), device="cuda")

    def loss():
        out, kept = layer.forward(x, B, T, zero.clone(), train=True)
        diff = out.double() - want.double()
        return float(0.5 * diff.square().sum()), kept, diff

    _, kept, diff = loss()
    grads, _ = layer.backward(kept, diff.bfloat16(), B, T)
    for n in ("q", "k", "v", "o"):
        W, d = layer.W[n], grads[n].float()
        step = 1e-2 * W.float().norm() / d.norm()
        values = []
        for sign in (1, -1):
            layer.W[n] = (W.float() + sign * step * d).bfloat16()
            moved = layer.W[n].double() - W.double()
            values.append((loss()[0], float((moved * d.double()).sum())))
        layer.W[n] = W
        want_change = values[0][1] - values[1][1]
        assert abs((values[0][0] - values[1][0]) - want_change) <= 0.15 * abs(want_change), n
