"""What a model has around its projected linear layers: the norms in front of them, the embedding and the log
probabilities at its two ends, and AdamW for the parameters that no projection covers (embeddings, output head, gains).

Like `layer.py` this owns buffers and issues library calls in order; every step is a HIP kernel
behind `grass.*`.  An object's buffers serve one stream, and one graph's replay, at a time.
"""
import torch

from . import grass
from .layer import AdamHyper

NORMS = {"layer": grass.NORM_LAYER, "rms": grass.NORM_RMS}


class NormLayer:
    """Layer norm or RMS norm over n features of up to T tokens, its parameters and their gradients (all
    fp32), and what a backward pass needs of the forward pass before it: one forward pass, whose X (where
    there is no R) is kept by reference and must not change until then; the next overwrites H, mean and rstd.  backward()
    writes the parameters' gradients and does not add to them: sums over several batches are the caller's."""

    def __init__(self, n, T, dtype, kind="rms", bias=False, eps=1e-5, device="cuda"):
        self.n, self.T, self.kind, self.eps = n, T, NORMS[kind], eps
        dt = grass.dtype_code(dtype)
        f32 = dict(dtype=torch.float32, device=device)
        self.gain, self.dgain = torch.ones(n, **f32), torch.zeros(n, **f32)
        self.bias = torch.zeros(n, **f32) if bias else None
        self.dbias = torch.zeros(n, **f32) if bias else None
        self.mean = torch.empty(T, **f32) if kind == "layer" else None
        self.rstd = torch.empty(T, **f32)
        # (shorter batches need no more: a workgroup leaves one row of sums, and there are no more of them)
        self.ws = grass.workspace(grass.norm_backward_workspace(T, n, dt), device)
        self.H = None

    def forward(self, X, R=None):
        """The norm of X (of X + R, the residual stream, which is kept as self.H) in a new tensor."""
        T, self.H = X.shape[0], None  # (a refused call leaves no pass to go backward from)
        assert T <= self.T
        Y, H = torch.empty_like(X), None if R is None else torch.empty_like(X)
        grass.norm_forward(X, self.gain, self.bias, self.eps, Y, self.kind, R=R, H=H,
                           mean=None if self.mean is None else self.mean[:T], rstd=self.rstd[:T])
        self.H = X if R is None else H
        return Y

    def backward(self, dY, dR=None):
        """The gradient of what forward() read, in a new tensor, plus dR, the residual stream's gradient from
        behind this layer; self.dgain and self.dbias receive the parameters' gradients."""
        assert self.H is not None, "no forward pass"
        T = dY.shape[0]
        dX = torch.empty_like(dY)
        return grass.norm_backward(dY, self.H, self.gain, None if self.mean is None else self.mean[:T], self.rstd[:T], dX,
                                   self.dgain, self.dbias, self.ws, self.kind, dR=dR)

    def parameters(self):
        """(weight, gradient) pairs."""
        return [(self.gain, self.dgain)] + ([(self.bias, self.dbias)] if self.bias is not None else [])


class Embedding:
    """The rows of E (V x n) by token, times `scale`, for up to T tokens at a time; dE: their gradient (a new fp32 tensor
    unless one is given: the head's, where it shares the weights).  Numbers outside 0 .. V - 1 are padding: rows of zeros,
    and no gradient.  backward() goes by the token numbers of the forward pass before it, which are kept by reference."""

    def __init__(self, E, T, scale=1.0, dE=None):
        V, n = E.shape
        self.E, self.T, self.scale, self.ids = E, T, scale, None
        self.dE = torch.zeros((V, n), dtype=torch.float32, device=E.device) if dE is None else dE
        # (by the gradient's rows the kernels tell tokens from padding: with fewer of them than E has, tokens would be lost)
        assert self.dE.shape == E.shape and self.dE.device == E.device, "the gradient has E's shape and device"
        grass.dtype_code(self.dE.dtype)
        self.ws = grass.workspace(grass.embed_backward_workspace(T, V, n), E.device)

    def forward(self, ids, dtype=None):
        """The tokens' rows in a new tensor of E's type, or of `dtype`."""
        T, self.ids = ids.shape[0], None  # (a refused call leaves no pass to go backward from)
        assert T <= self.T
        Y = torch.empty((T, self.E.shape[1]), dtype=dtype or self.E.dtype, device=self.E.device)
        grass.embed_forward(self.E, ids, Y, self.scale)
        self.ids = ids
        return Y

    def backward(self, dY, accumulate=False):
        """self.dE from the gradient of what forward() gave; added to what it holds where accumulate is true."""
        assert self.ids is not None, "no forward pass"
        return grass.embed_backward(dY, self.ids, self.dE, self.ws, self.scale, accumulate)

    def parameters(self):
        """(weight, gradient) pairs."""
        return [(self.E, self.dE)]


class TokenLoss:
    """Log probabilities of given tokens under up to T rows of V logits of type `dtype`, and the gradient of a loss made of
    them.  scale: the inverse of a temperature.  backward() goes by the logits and targets of the forward pass before it, which
    are kept by reference.  Targets outside 0 .. V - 1 are padding: log probability 0, and no gradient."""

    def __init__(self, T, V, dtype, scale=1.0, device="cuda"):
        self.T, self.scale = T, scale
        f32 = dict(dtype=torch.float32, device=device)
        self.logp, self.rmax, self.rlog, self.entropy = (torch.empty(T, **f32) for _ in range(4))
        self.ws = grass.workspace(grass.logp_forward_workspace(T, V, 0, grass.dtype_code(dtype)), device)
        self.given = None

    def forward(self, logits, targets, entropy=False):
        """The targets' log probabilities (and the rows' entropies): views that the next forward pass writes over."""
        T, self.given = logits.shape[0], None  # (a refused call leaves no pass to go backward from)
        assert T <= self.T
        logp, H = self.logp[:T], self.entropy[:T] if entropy else None
        grass.logp_forward(logits, targets, logp, self.ws, self.scale, entropy=H, rmax=self.rmax[:T], rlog=self.rlog[:T])
        self.given = logits, targets, entropy
        return (logp, H) if entropy else logp

    def backward(self, dlogp, dentropy=None, in_place=True):
        """The gradient of the logits from that of logp (and of the entropies, if forward() gave them): written over the
        logits, so that it is had once, or into a new tensor."""
        assert self.given is not None, "no forward pass, or its logits are written over"
        logits, targets, entropy = self.given
        assert dentropy is None or entropy, "the forward pass left no entropies"
        T = logits.shape[0]
        dlogits = grass.logp_backward(logits, targets, self.rmax[:T], self.rlog[:T], dlogp,
                                      logits if in_place else torch.empty_like(logits), self.scale,
                                      entropy=self.entropy[:T] if dentropy is not None else None, dentropy=dentropy)
        if in_place:
            self.given = None
        return dlogits


class AdamW:
    """AdamW over (weight, gradient) pairs whose tensors stay where they are.  moments: "f32", or "q8" for
    8-bit moments of the tensors of at least `least_q8` elements (small ones, gains above all, keep
    fp32: they cost nothing); of 128 consecutive elements, those whose gradients stay some 30000 times smaller than the
    largest ones' take steps that are too short.  weight_decay applies to matrices.  max_norm: the gradients' global
    norm is clipped to it, and a step whose
    gradients are not finite changes nothing (t counts it all the same).  The gradients are to be written into the
    same tensors each step: laying a plan out takes the host 2 us a tensor (300 of them 0.7 ms), much more than a step."""

    def __init__(self, parameters, adam=None, weight_decay=0.0, moments="f32", least_q8=4096, max_norm=None):
        assert moments in ("f32", "q8")
        self.adam, self.max_norm, self.t = adam or AdamHyper(), max_norm, 0
        W, G = [p[0] for p in parameters], [p[1] for p in parameters]
        self.M, self.V, self.Mscale, self.Vscale = [], [], [], []
        for w in W:
            n, dev = w.numel(), w.device
            q8 = moments == "q8" and n >= least_q8
            for into, scales, dtype in ((self.M, self.Mscale, torch.float8_e4m3fn), (self.V, self.Vscale, torch.float8_e5m2)):
                into.append(torch.zeros(n, dtype=torch.uint8, device=dev).view(dtype) if q8 else
                            torch.zeros(n, dtype=torch.float32, device=dev))
                scales.append(torch.ones(grass.moment_blocks(n), dtype=torch.float32, device=dev) if q8 else None)
        self.plan = grass.adamw_plan(W, G, self.M, self.V, [weight_decay if w.dim() > 1 else 0.0 for w in W],
                                     self.Mscale, self.Vscale)
        dev = W[0].device if W else "cuda"
        self.norm = torch.zeros(2, dtype=torch.float32, device=dev)  # of the last step's gradients, and their factor
        self.ws = grass.workspace(grass.grad_norm_workspace(self.plan), dev)

    def step(self, lr=None, step_scalars=None):
        """One step; step_scalars: see grass.adamw_step (the caller counts the steps of a captured one)."""
        a, scale = self.adam, None
        if self.max_norm is not None:
            grass.grad_norm(self.plan, self.max_norm, self.norm, self.ws)
            scale = self.norm[1:]
        if step_scalars is None:
            self.t += 1
        grass.adamw_step(self.plan, a.lr if lr is None else lr, a.beta1, a.beta2, a.eps, max(self.t, 1), grad_scale=scale,
                         step_scalars=step_scalars)
