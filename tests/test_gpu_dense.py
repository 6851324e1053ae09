"""The drivers around the norms and AdamW, and the example that runs them beside GRASS layers."""
import importlib.util
import math
import os

import pytest
import torch

from gpu_util import DEV
from paper_2406_17660_amd.dense import AdamW, NormLayer
from paper_2406_17660_amd.layer import AdamHyper

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_learns():
    spec = importlib.util.spec_from_file_location("train_tiny", os.path.join(ROOT, "examples", "train_tiny.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(200)
    assert all(math.isfinite(x) for x in losses)
    assert abs(losses[0] - math.log(512)) < 0.5 and sum(losses[-10:]) / 10 < 0.5 * math.log(512)


@pytest.mark.parametrize("kind,bias", [("layer", True), ("rms", False)])
def test_norm_layer_against_autograd(kind, bias):
    """Two norms with a residual branch between them, in fp32, against torch's automatic gradients in 64 bits
    (all within 1e-5 of the largest value: some hundred fp32 roundings)."""
    T, n = 33, 120
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    X, dY = (torch.randn((T, n), generator=g, device=DEV) for _ in range(2))
    a, b = (NormLayer(n, T + 5, torch.float32, kind, bias) for _ in range(2))
    for layer in (a, b):
        layer.gain.copy_(1 + 0.2 * torch.randn(n, generator=g, device=DEV))
    Y = b.forward(a.forward(X), R=X)
    dH = b.backward(dY)
    dX = a.backward(dH, dR=dH)

    def plain(h, gain, beta):
        d = h - h.mean(1, keepdim=True) if kind == "layer" else h
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gain
        return y + beta if bias else y

    x, ga, gb = (t.double().cpu().requires_grad_() for t in (X, a.gain, b.gain))
    ba, bb = (torch.zeros(n, dtype=torch.float64, requires_grad=True) for _ in range(2))
    y = plain(plain(x, ga, ba) + x, gb, bb)
    y.backward(dY.double().cpu())
    pairs = [(Y, y.detach()), (dX, x.grad), (a.dgain, ga.grad), (b.dgain, gb.grad)]
    pairs += [(a.dbias, ba.grad), (b.dbias, bb.grad)] if bias else []
    for got, want in pairs:
        assert float((got.double().cpu() - want).abs().max()) <= 1e-5 * float(want.abs().max())


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_adamw_finds_a_minimum_and_skips_what_is_not_finite(moments):
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    target = [torch.randn(s, generator=g, device=DEV) for s in ((64, 200), (7,))]
    W = [torch.zeros_like(t) for t in target]
    G = [torch.zeros_like(t) for t in target]
    opt = AdamW(list(zip(W, G)), AdamHyper(lr=0.05), moments=moments, max_norm=10.0)
    for t in range(400):
        for w, d, x in zip(W, G, target):
            d.copy_(w - x)
        opt.step(lr=0.05 * (1 - t / 400))
    assert all(float((w - x).abs().max()) < 0.02 for w, x in zip(W, target))
    G[1][3] = float("nan")
    was = [w.clone() for w in W]
    opt.step()
    assert math.isnan(opt.norm[1].item()) and all(torch.equal(a, b) for a, b in zip(W, was))
