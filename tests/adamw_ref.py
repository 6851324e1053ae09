"""AdamW with fp32 and 8-bit moments on the CPU, from the formulas of include/grass.h: the moments with
fp32's rounding after every product and sum (numpy's own fp32), the codes by arithmetic in 64 bits."""
import numpy as np

BLOCK = 128
f = np.float32


def moments(g, scale, m, v, b1, b2):
    """New m and v (float32 arrays)."""
    with np.errstate(all="ignore"):
        b1, b2 = f(b1), f(b2)
        x = g.astype(f) * f(scale)
        return b1 * m + (f(1) - b1) * x, b2 * v + ((f(1) - b2) * x) * x


def update(w, m, v, lr, b1, b2, eps, t, decay):
    """The new weights in 64 bits, and the magnitudes that enter them."""
    with np.errstate(all="ignore"):
        lr, b1, b2, eps = (float(f(x)) for x in (lr, b1, b2, eps))
        step = lr * (m.astype(np.float64) / (1 - b1 ** t)) / (np.sqrt(v.astype(np.float64) / (1 - b2 ** t)) + eps)
        keep = 1 - lr * float(f(decay))
        w = w.astype(np.float64)
        return w * keep - step, np.abs(w) + np.abs(step)


KIND = {"M": (3, 7, -6, 0x6A09E667), "V": (2, 14, -14, 0xBB67AE85)}  # mantissa bits, scale, least exponent, thresholds


def encode(x, t, kind):
    """Codes (uint8) and scales (float32) of a tensor's moment x (1-D float32) after step t."""
    man, top, low, multiple = KIND[kind]
    n = x.size
    nb = -(-n // BLOCK)
    pad = np.zeros(nb * BLOCK, np.float64)
    pad[:n] = x
    pad = pad.reshape(nb, BLOCK)
    fine = np.isfinite(pad)
    a = np.where(fine, np.abs(pad), 0.0)
    amax = a.max(1, initial=0.0)
    e = np.where(amax > 0, np.frexp(amax)[1] - 1, -103)
    e = np.maximum(e, -103)
    scale = np.ldexp(1.0, e - top)
    a = a / scale[:, None]
    k = np.maximum(np.where(a > 0, np.frexp(a)[1] - 1, low), low)
    bits = 23 - man
    j = np.arange(BLOCK, dtype=np.uint64)
    word = (j * np.uint64(0x9E3779B1) + np.uint64((t % (1 << 24)) * multiple)) % np.uint64(1 << 32)
    u = (word >> np.uint64(32 - bits)).astype(np.float64) / 2.0 ** bits
    # multiples of the step, after fp32's own rounding where the type's numbers are subnormal
    q = np.floor(np.rint(np.ldexp(a, man - k + bits)) / 2.0 ** bits + u)
    # q steps of 2^(k - man) as a code: q < 2^man only where k = low (the subnormal numbers, exponent field 0)
    code = (k - low) * 2 ** man + q
    if kind == "V":  # what is not zero is not stored as zero
        code = np.maximum(code, pad != 0)
    code = np.where(fine, code, 127).astype(np.uint8) | np.where(np.signbit(pad), 128, 0).astype(np.uint8)
    return code.reshape(-1)[:n], scale.astype(f)


def decode(code, scale, kind):
    """The fp32 values of codes and scales."""
    man, top, low, _ = KIND[kind]
    c = code.astype(np.int64)
    body, sign = c & 127, np.where(c & 128, -1.0, 1.0)
    field, frac = body >> man, body & (2 ** man - 1)
    value = np.where(field > 0, np.ldexp(1.0 + frac / 2.0 ** man, field - 1 + low), np.ldexp(frac / 2.0 ** man, low))
    if kind == "M":
        value = np.where(body == 127, np.nan, value)
    else:
        value = np.where(field == 31, np.where(frac > 0, np.nan, np.inf), value)
    return (sign * value * np.repeat(scale.astype(np.float64), BLOCK)[:c.size]).astype(f)
