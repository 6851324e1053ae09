"""The 64-bit references of the embedding and of the log probabilities, against automatic differentiation and
differences (CPU only)."""
import numpy as np
import torch

import ends_ref


def test_embedding_against_automatic_gradients():
    g = torch.Generator().manual_seed(1)
    E = torch.randn((7, 5), generator=g, dtype=torch.float64, requires_grad=True)
    ids = torch.tensor([3, 3, 0, 6, 3, -1, 7, 1 << 40])
    dY = torch.randn((8, 5), generator=g, dtype=torch.float64)
    there = (ids >= 0) & (ids < 7)
    Y = E[torch.where(there, ids, 0)] * 1.5 * there[:, None]
    Y.backward(dY)
    assert np.allclose(ends_ref.embed_forward(E.detach().numpy(), ids.numpy(), 1.5), Y.detach().numpy(), rtol=1e-14)
    dE, size, count = ends_ref.embed_backward(dY.numpy(), ids.numpy(), 7, 1.5)
    assert np.allclose(dE, E.grad.numpy(), rtol=1e-13, atol=1e-14)
    assert count.tolist() == [1, 0, 0, 3, 0, 0, 1] and (size >= np.abs(dE) - 1e-14).all()


def rows():
    x = np.random.default_rng(2).normal(0, 2, (6, 11))
    x[1, 3:] = -np.inf
    x[2] = -np.inf
    x[3, 4] = np.nan
    x[4, 4] = np.inf
    x[5] = 1.25
    return x


def test_log_probabilities_and_special_rows():
    x, scale = rows(), 0.7
    m, rlog, logp, H = ends_ref.logp_rows(x, scale)
    fine = [0, 1, 5]
    want = torch.log_softmax(torch.tensor(x[fine]) * scale, 1)
    assert np.allclose(logp[fine], want.numpy(), rtol=1e-13)
    assert np.allclose(H[fine], torch.special.entr(want.exp()).sum(1).numpy(), rtol=1e-12)
    assert np.allclose((m * scale + rlog)[fine], torch.logsumexp(torch.tensor(x[fine]) * scale, 1).numpy(), rtol=1e-13)
    assert m[2] == -np.inf and rlog[2] == 0 and H[2] == 0 and (logp[2] == -np.inf).all()
    assert np.isnan(rlog[3:5]).all() and np.isnan(H[3:5]).all() and np.isnan(logp[3:5]).all()
    idx, val = ends_ref.alternatives(x, logp, 4)
    assert idx[5].tolist() == [0, 1, 2, 3] and idx[2].tolist() == [-1] * 4 and (val[2] == -np.inf).all()
    assert sorted(idx[1].tolist()) == [-1, 0, 1, 2] and val[1, 3] == -np.inf and np.isnan(val[3:5]).all() and (idx[3:5] == -1).all()
    assert ends_ref.given(logp, np.array([1, 5, 0, -1, 11, 2])).tolist()[1:5] == [-np.inf, -np.inf, 0, 0]


def test_gradient_against_automatic_gradients_and_differences():
    x, scale = rows()[[0, 1, 2, 5, 0]], 0.7
    targets = np.array([3, 1, 0, 10, -100])
    rng = np.random.default_rng(3)
    dlogp, dH = rng.normal(size=5), rng.normal(size=5)
    m, rlog, logp, H = ends_ref.logp_rows(x, scale)
    got, _, _ = ends_ref.logp_backward(x, targets, scale, m, rlog, dlogp, H, dH)
    assert (got[2] == 0).all() and (got[1, 3:] == 0).all()

    def loss(z):
        _, _, l, h = ends_ref.logp_rows(z, scale)
        return (ends_ref.given(l, targets) * dlogp + h * dH)

    for t, j in ((0, 3), (0, 4), (1, 1), (1, 2), (3, 10), (3, 0), (4, 6)):
        step = np.zeros_like(x)
        step[t, j] = 1e-5
        slope = (loss(x + step)[t] - loss(x - step)[t]) / 2e-5
        assert abs(slope - got[t, j]) < 1e-8 * (1 + abs(slope)), (t, j)
    z = torch.tensor(x[[0, 3]], requires_grad=True)
    l = torch.log_softmax(z * scale, 1)
    (l[[0, 1], [3, 10]] * torch.tensor(dlogp[[0, 3]]) - (l.exp() * l).sum(1) * torch.tensor(dH[[0, 3]])).sum().backward()
    assert np.allclose(got[[0, 3]], z.grad.numpy(), rtol=1e-12, atol=1e-15)
