"""Layer norm and RMS norm in 64 bits, as the tests of the HIP kernels use them (numpy, CPU)."""
import numpy as np


def forward(h, gain, bias, eps, centre):
    """y, mean, rstd of the rows of h (float64); gain, bias: float64 or None."""
    mean = h.mean(1) if centre else np.zeros(h.shape[0])
    d = h - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    if gain is not None:
        y = y * gain
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def backward(dy, h, gain, mean, rstd, centre):
    """dx, dgain, dbias for the statistics that the forward pass kept."""
    xh = (h - mean[:, None] if centre else h) * rstd[:, None]
    z = dy if gain is None else dy * gain
    dx = z - xh * (z * xh).mean(1)[:, None]
    if centre:
        dx = dx - z.mean(1)[:, None]
    return dx * rstd[:, None], (dy * xh).sum(0), dy.sum(0)
