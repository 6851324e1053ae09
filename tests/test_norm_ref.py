"""The 64-bit norm that the GPU tests compare with: its gradients against central differences."""
import numpy as np
import pytest

import norm_ref


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("T,n", [(1, 1), (3, 2), (4, 7), (2, 33)])
def test_backward_is_the_derivative_of_forward(centre, T, n):
    rng = np.random.default_rng(T * 100 + n)
    h, dy = rng.normal(size=(T, n)) + 0.3, rng.normal(size=(T, n))
    gain, bias, eps = 1 + 0.1 * rng.normal(size=n), rng.normal(size=n), 1e-2

    def loss(h, gain, bias):
        return float((norm_ref.forward(h, gain, bias, eps, centre)[0] * dy).sum())

    _, mean, rstd = norm_ref.forward(h, gain, bias, eps, centre)
    got = norm_ref.backward(dy, h, gain, mean, rstd, centre)
    step = 1e-5  # central differences: about step^2 off, and rounding / step
    for k, want_of in enumerate((h, gain, bias)):
        want = np.zeros_like(want_of)
        for at in np.ndindex(want_of.shape):
            args = [h.copy(), gain.copy(), bias.copy()]
            args[k][at] += step
            up = loss(*args)
            args[k][at] -= 2 * step
            want[at] = (up - loss(*args)) / (2 * step)
        assert np.allclose(got[k], want, rtol=1e-6, atol=1e-6)
