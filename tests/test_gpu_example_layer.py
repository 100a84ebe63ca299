"""The example's training step against 64-bit autograd of the same layer, and its training.

The step's roundings: int8 codes of n and dout (step amax / 127 of a row, amax about 3.5 times
the row's rms, so 3.5 / 127 / sqrt(12) = 0.8 % of a row's norm each), int8 block codes of the
saved n (less: blocks of 128), bf16 storage (0.2 %).  A gradient gathers two or three of
these, independent: under 1.5 %, and twice that is allowed.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(hl):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "adapter_layer.py")
    spec = importlib.util.spec_from_file_location("adapter_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("tokens,width,channels", [(1, 128, 64), (37, 256, 144), (300, 896, 528)])
def test_gradients(example, tokens, width, channels):
    layer = example.AdapterLayer(tokens, width, channels, seed=tokens)
    g = torch.Generator(device="cuda").manual_seed(7)
    for t in (layer.res, layer.y, layer.dout):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    for t, sigma in ((layer.b, 0.1), (layer.w_pre, 0.1), (layer.gate, 0.3)):
        t.p16.add_(sigma * torch.randn(t.p16.shape, generator=g, device="cuda"))
    layer.forward()
    layer.backward()

    d = {k: getattr(layer, k).p16.cpu().double().requires_grad_() for k in ("a", "b", "w_pre", "gate")}
    res, y = (getattr(layer, k).cpu().double().requires_grad_() for k in ("res", "y"))
    w = layer.w.cpu().double() * layer.w_scales.cpu().double()[:, None]
    h = res + d["gate"] * y
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * d["w_pre"]
    out = n @ w.t() + layer.s * (n @ d["a"].t()) @ d["b"].t()
    out.backward(layer.dout.cpu().double())

    def off(got, want):
        want = want.detach()
        return float((got.cpu().double().reshape(want.shape) - want).norm() / want.norm())

    assert off(layer.out, out) < 0.03
    found = {k: off(getattr(layer, k).grad, d[k].grad) for k in d}
    found |= {"res": off(layer.dres, res.grad), "y": off(layer.dy, y.grad)}
    assert max(found.values()) < 0.03, found


def test_training_learns(example):
    losses = example.train(tokens=256, width=256, channels=272, steps=60)
    assert losses[-1] < 0.25 * losses[0], (losses[0], losses[-1])
    assert losses == example.train(tokens=256, width=256, channels=272, steps=60)  # the same bits again
