"""The drivers around the norms and AdamW, and the example that runs them beside GRASS layers."""
import importlib.util
import math
import os

import pytest
import torch

from gpu_util import DEV
from paper_2406_17660_amd.dense import AdamW, Embedding, NormLayer, TokenLoss
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


@pytest.mark.parametrize("shared", [False, True])
def test_embedding_and_loss_against_autograd(shared):
    """A model of an embedding, a norm and a head (the embedding itself, or one of its own), in fp32, against torch's
    automatic gradients in 64 bits; padding among tokens and targets, an entropy bonus, a batch shorter than the layers are
    made for.  All within 1e-5 of the largest value: some hundred fp32 roundings."""
    T, V, n, scale = 41, 30, 24, 3.0
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    E, head = (torch.randn((V, n), generator=g, device=DEV) * 0.3 for _ in range(2))
    head = E if shared else head
    tokens, targets = (torch.randint(V, (T,), generator=g, device=DEV) for _ in range(2))
    tokens[3], targets[5], targets[6] = -1, -100, V
    dlogp, dH = torch.randn(T, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)
    dhead = torch.empty((V, n), device=DEV)
    embedding = Embedding(E, T + 9, scale, dE=dhead if shared else None)
    norm, loss = NormLayer(n, T + 9, torch.float32, "rms"), TokenLoss(T + 9, V, torch.float32, 0.8)
    y = norm.forward(embedding.forward(tokens))
    logits = y @ head.t()
    logp, H = loss.forward(logits, targets, entropy=True)
    logp, H = logp.clone(), H.clone()
    kept = loss.backward(dlogp, dH, in_place=False)
    dlogits = loss.backward(dlogp, dH)
    assert torch.equal(kept, dlogits) and dlogits.data_ptr() == logits.data_ptr()
    with pytest.raises(AssertionError):  # the logits are gone
        loss.backward(dlogp, dH)
    torch.mm(dlogits.t(), y, out=dhead)
    embedding.backward(norm.backward(dlogits @ head), accumulate=shared)

    e = E.double().cpu().requires_grad_()
    w = e if shared else head.double().cpu().requires_grad_()
    t, j = tokens.cpu(), targets.cpu()
    there = (t >= 0).view(-1, 1)
    x = e[t.clamp(min=0)] * scale * there
    z = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)
    l = torch.log_softmax(z @ w.t() * 0.8, 1)
    counted = ((j >= 0) & (j < V)).double()
    want_logp = l.gather(1, j.clamp(0, V - 1).view(-1, 1))[:, 0] * counted
    want_H = -(l.exp() * l).sum(1)
    (want_logp @ dlogp.double().cpu() + want_H @ dH.double().cpu()).backward()
    pairs = [(logp, want_logp), (H, want_H), (embedding.dE, e.grad)] + ([] if shared else [(dhead, w.grad)])
    for got, want in pairs:
        assert float((got.double().cpu() - want.detach()).abs().max()) <= 1e-5 * float(want.detach().abs().max())


def test_a_training_step_of_the_example_in_a_graph():
    """The calls of the ends of a model one behind the other, captured, and replayed with other tokens."""
    T, V, n = 300, 500, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    E, head = ((torch.randn((V, n), generator=g, device=DEV) * 0.1).bfloat16() for _ in range(2))
    embedding, loss = Embedding(E, T), TokenLoss(T, V, torch.bfloat16)
    dlogp = torch.full((T,), -1.0 / T, device=DEV)
    tokens, targets, wT = torch.zeros(T, dtype=torch.int64, device=DEV), torch.zeros(T, dtype=torch.int64, device=DEV), head.t().contiguous()
    out = {}

    def step():
        h = embedding.forward(tokens)
        out["logp"] = loss.forward(h @ wT, targets)
        out["dE"] = embedding.backward(loss.backward(dlogp) @ head)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        for ids in (tokens, targets):
            ids.copy_(torch.randint(-2, V + 2, (T,), generator=g, device=DEV))
        embedding.dE.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = {k: v.clone() for k, v in out.items()}
        assert not torch.isnan(replayed["dE"]).any()
        step()
        assert all(torch.equal(out[k], replayed[k]) for k in out)
