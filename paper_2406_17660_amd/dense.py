"""What a model has around its projected linear layers: the norms in front of them, and AdamW for the
parameters that no projection covers (embeddings, output head, gains).

Like `layer.py` this owns buffers and issues library calls in order; every step is a HIP kernel
behind `grass.*`.
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
        dt = grass.F32 if dtype == torch.float32 else grass.BF16
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
        T = X.shape[0]
        assert T <= self.T
        Y = torch.empty_like(X)
        self.H = X if R is None else torch.empty_like(X)
        grass.norm_forward(X, self.gain, self.bias, self.eps, Y, self.kind, R=R, H=None if R is None else self.H,
                           mean=None if self.mean is None else self.mean[:T], rstd=self.rstd[:T])
        return Y

    def backward(self, dY, dR=None):
        """The gradient of what forward() read, in a new tensor, plus dR, the residual stream's gradient from
        behind this layer; self.dgain and self.dbias receive the parameters' gradients."""
        T = dY.shape[0]
        dX = torch.empty_like(dY)
        return grass.norm_backward(dY, self.H, self.gain, None if self.mean is None else self.mean[:T], self.rstd[:T], dX,
                                   self.dgain, self.dbias, self.ws, self.kind, dR=dR)

    def parameters(self):
        """(weight, gradient) pairs."""
        return [(self.gain, self.dgain)] + ([(self.bias, self.dbias)] if self.bias is not None else [])


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
