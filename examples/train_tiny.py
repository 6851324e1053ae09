"""A small language model trained with everything the package has: the linear layers of its MLP by GRASS
steps on r of their rows, embedding, output head and gains by AdamW with 8-bit moments and clipping,
the norms and their gradients in between, the embedding lookup and the loss at its ends.

    python examples/train_tiny.py [steps]

The text is synthetic: token t + 1 is a fixed permutation of token t, one time in ten any token, so
that the loss can fall from ln(vocabulary) to about 0.1 ln(vocabulary) + 0.33.  Matrix products of the
forward pass are torch's; there is no autograd.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2406_17660_amd import grass  # noqa: E402
from paper_2406_17660_amd.dense import AdamW, Embedding, NormLayer, TokenLoss  # noqa: E402
from paper_2406_17660_amd.layer import AdamHyper, GrassLayer  # noqa: E402

DEV, BF16 = "cuda", torch.bfloat16


class TinyModel:
    def __init__(self, vocab=512, hidden=256, inner=688, T=2048, r=64, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        normal = lambda *shape: (torch.randn(shape, generator=g, device=DEV) * 0.05).to(BF16)  # noqa: E731
        self.T, self.vocab = T, vocab
        self.embedding, self.head = Embedding(normal(vocab, hidden), T), normal(vocab, hidden)
        self.loss = TokenLoss(T, vocab, BF16)
        self.dlogp = torch.full((T,), -1.0 / T, device=DEV)  # of the mean over the tokens
        self.up, self.down = normal(inner, hidden), normal(hidden, inner)
        self.norm1, self.norm2 = (NormLayer(hidden, T, BF16, kind) for kind in ("rms", "rms"))
        self.dhead = torch.empty((vocab, hidden), device=DEV)
        self.ws_head = grass.workspace(grass.dense_workspace(T, vocab, hidden, grass.BF16))
        adam = AdamHyper(lr=3e-3)
        self.grass = {name: GrassLayer(m, n, r, T, BF16, "multi_norm", True, alpha=1.0, adam=adam, seed=seed + k)
                      for k, (name, (m, n)) in enumerate({"up": (inner, hidden), "down": (hidden, inner)}.items())}
        self.adamw = AdamW(self.embedding.parameters() + [(self.head, self.dhead)] + self.norm1.parameters() + self.norm2.parameters(),
                           adam, weight_decay=0.01, moments="q8", max_norm=1.0)
        self.t = 0

    def step(self, tokens, targets, refresh_every=20):
        """Forward pass, backward pass and update; returns the loss (on the device)."""
        h0 = self.embedding.forward(tokens)
        y1 = self.norm1.forward(h0)
        a = y1 @ self.up.t()
        act = torch.relu(a)
        y2 = self.norm2.forward(act @ self.down.t(), R=h0)
        loss = -self.loss.forward(y2 @ self.head.t(), targets).mean()

        dlogits = self.loss.backward(self.dlogp)
        grass.dense_grad(dlogits, y2, self.dhead, self.ws_head)
        dh1 = self.norm2.backward(dlogits @ self.head)
        da = (dh1 @ self.down) * (a > 0)
        dh0 = self.norm1.backward(da @ self.up, dR=dh1)
        self.embedding.backward(dh0)

        for name, dY, X, W in (("down", dh1, act, self.down), ("up", da, y1, self.up)):
            layer = self.grass[name]
            if self.t % refresh_every == 0:
                layer.refresh_step(dY, X, W)
            else:
                layer.step(dY, X, W)
        self.adamw.step()
        self.t += 1
        return loss


def batch(model, permutation, generator):
    """Tokens and the ones that follow them."""
    tokens = torch.randint(model.vocab, (model.T,), generator=generator, device=DEV)
    anything = torch.randint(model.vocab, (model.T,), generator=generator, device=DEV)
    other = torch.rand(model.T, generator=generator, device=DEV) < 0.1
    return tokens, torch.where(other, anything, permutation[tokens])


def train(steps=300, report=None):
    """Losses of a run."""
    model = TinyModel()
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    permutation = torch.randperm(model.vocab, generator=g, device=DEV)
    losses = []
    for t in range(steps):
        losses.append(model.step(*batch(model, permutation, g)))
        if report and t % 50 == 0:
            report(f"step {t}: loss {losses[-1].item():.3f}, norm of the dense gradients {model.adamw.norm[0].item():.3f}")
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    run = train(int(sys.argv[1]) if len(sys.argv) > 1 else 300, print)
    print(f"loss {run[0]:.3f} (ln of the vocabulary: {math.log(512):.3f}) -> {sum(run[-10:]) / len(run[-10:]):.3f}")
