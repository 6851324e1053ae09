"""The two ends of a model in 64 bits, as the tests of the HIP kernels use them (numpy, CPU): the embedding
lookup and its gradient, log probabilities of given tokens with entropy and alternatives, and their
gradient."""
import numpy as np


def embed_forward(E, ids, scale):
    out = np.zeros((len(ids), E.shape[1]))
    there = (ids >= 0) & (ids < E.shape[0])
    out[there] = E[ids[there]] * scale
    return out


def embed_backward(dY, ids, V, scale):
    """The gradient, and per row the sum of magnitudes and the number of terms (for tolerances)."""
    out, size, count = np.zeros((V, dY.shape[1])), np.zeros((V, dY.shape[1])), np.zeros(V, np.int64)
    there = (ids >= 0) & (ids < V)
    np.add.at(out, ids[there], dY[there] * scale)
    np.add.at(size, ids[there], np.abs(dY[there] * scale))
    np.add.at(count, ids[there], 1)
    return out, size, count


def logp_rows(x, scale):
    """rmax, rlog, log p (T x V) and entropy.  Rows that are all masked: -inf, 0, -inf and 0; with NaN or +inf: NaN."""
    with np.errstate(all="ignore"):
        m = np.where(np.isnan(x), -np.inf, x).max(1)
        spoiled = np.isnan(x).any(1) | (m == np.inf)
        none = (x == -np.inf).all(1)
        d = (x - np.where(np.isfinite(m), m, 0.0)[:, None]) * scale
        e = np.exp(d)
        rlog = np.where(none, 0.0, np.log(np.where(none, 1.0, e.sum(1))))
        rlog[spoiled] = np.nan
        logp = np.where(none[:, None], -np.inf, d - rlog[:, None])
        p = np.exp(logp)
        entropy = -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0).sum(1)
        logp[spoiled], entropy[spoiled] = np.nan, np.nan
    return m, rlog, logp, entropy


def given(logp, targets):
    out = np.zeros(len(targets))
    there = (targets >= 0) & (targets < logp.shape[1])
    out[there] = logp[there, targets[there]]
    return out


def alternatives(x, logp, top):
    """Tokens of the largest logits (ties: the lower one) and their log probabilities; -1 and -inf where no more have a
    probability, -1 and NaN in rows with a NaN or +inf."""
    T, V = x.shape
    idx, val = np.full((T, top), -1, np.int64), np.full((T, top), -np.inf)
    for t in range(T):
        if np.isnan(x[t]).any() or (x[t] == np.inf).any():
            val[t] = np.nan
            continue
        order = np.lexsort((np.arange(V), -x[t]))[:top]
        order = order[x[t, order] > -np.inf]
        idx[t, :len(order)], val[t, :len(order)] = order, logp[t, order]
    return idx, val


def logp_backward(x, targets, scale, rmax, rlog, dlogp, entropy, dentropy):
    """The gradient of the logits, and log p and p as rmax and rlog give them."""
    with np.errstate(all="ignore"):
        l = (x - np.where(rmax == -np.inf, 0.0, rmax)[:, None]) * scale - rlog[:, None]
        p = np.exp(l)
        masked = (rmax == -np.inf) & (rlog == 0)
        there = (targets >= 0) & (targets < x.shape[1]) & ~masked
        g = np.where(there, dlogp, 0.0)
        out = -g[:, None] * p
        out[there, targets[there]] += g[there]
        out -= np.where(p == 0, 0.0, dentropy[:, None] * p * (l + entropy[:, None]))
        out[(g == 0) & (dentropy == 0)] = 0.0
    return out * scale, l, p
