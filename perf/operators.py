"""The operators of a training step around the projected linear layers, as timed cases: the norms in
front of the linear layers (forward and backward), the global norm of the gradients with its clipping
factor, and the AdamW step over all the tensors that no projection covers (embeddings, output head,
gains), with moments in 32 bits or in 8.

A case is a dict of plain values:

  kind      "forward", "backward", "adamw" or "grad_norm"
  T, n      tokens and features of a norm
  norm      "layer" (mean and variance) or "rms"
  dtype     type of the activations ("bf16" or "f32"); of the weights in "adamw" and "grad_norm"
  gdtype    type of gain and bias; of the gradients in "adamw" and "grad_norm"
  add       forward: a residual branch is added first, and the sum stored; backward: the gradient
            that reaches that sum by its other way is added
  bias      the norm has a bias
  serve     forward: the statistics are not kept, as where no backward pass follows
  tensors   "gains": `count` gains of `hidden`; "model": embedding and head of `vocab` rows and
            `count` gains of `hidden`; "ragged": `count` sizes up to `most` from the seed `pick`
  moments   "f32" or "q8" (8 bits with a scale for each 128 elements)

The 8-bit moments: M holds e4m3 and V e5m2 values, each block of 128 elements with a power of two as
its scale, 2^(e-7) and 2^(e-14) for the largest finite value's exponent e (at least -103).  A new
moment is formed in fp32, each product and sum rounded by itself, and divided by its block's new
scale; it becomes a multiple of the type's step there by floor(x / step + u), u from [0, 1) by the
element's place in its block and the step number, so that what a step loses another one gains.
Anything that is not finite is stored as NaN.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
# A step in the middle of a run: the moments are warm.
ADAM_T = 1000
MAX_NORM = 1.0
GRAD_SCALE = 0.37  # what clipping left of this step's gradients
BLOCK = 128
MOST_ACTIVATIONS = 131072 * 4096  # a drawn case stays under the largest listed ones
MOST_ELEMENTS = 2 * 32000 * 4096


def _norm(name, kind, T, n, norm, dtype, gdtype, add=False, bias=False, serve=False):
    case = {"kind": kind, "T": T, "n": n, "norm": norm, "dtype": dtype, "gdtype": gdtype, "add": add, "bias": bias}
    if kind == "forward":
        case["serve"] = serve
    return {"name": name, **case} if name else case


def _tensors(name, kind, tensors, dtype, gdtype, moments=None, **sizes):
    case = {"kind": kind, "tensors": tensors, "dtype": dtype, "gdtype": gdtype, **sizes}
    if kind == "adamw":
        case["moments"] = moments
    return {"name": name, **case} if name else case


def listed():
    return [
        # One token through the norm in front of a 7B layer, with the residual sum: latency.
        _norm("forward_token", "forward", 1, 4096, "rms", "bf16", "bf16", add=True, serve=True),
        # A 7B block's norm over the full token batch.
        _norm("forward_7b", "forward", 131072, 4096, "rms", "bf16", "bf16", add=True),
        # An odd width and a batch as long as its texts, in reference precision.
        _norm("forward_odd", "forward", 2407, 1293, "layer", "f32", "f32", bias=True),
        # The smallest model's norm in training: short rows, many of them.
        _norm("backward_60m", "backward", 65536, 512, "layer", "bf16", "f32", bias=True),
        # A 7B block's norm over the full token batch.
        _norm("backward_7b", "backward", 131072, 4096, "rms", "bf16", "bf16", add=True),
        # One short batch in fine-tuning, at the 1B model's odd inner width.
        _norm("backward_odd", "backward", 2047, 5461, "layer", "bf16", "f32", bias=True),
        # The gains of a 7B model alone: many small tensors, where launches count.
        _tensors("adamw_gains_7b", "adamw", "gains", "f32", "f32", "f32", count=65, hidden=4096),
        # Everything of a 350M model that is not projected, moments in 32 bits.
        _tensors("adamw_350m", "adamw", "model", "bf16", "bf16", "f32", count=49, hidden=1024, vocab=32000),
        # Many tensors of any size one behind the other in one buffer, so that few start on 16 bytes.
        _tensors("adamw_ragged_q8", "adamw", "ragged", "bf16", "f32", "q8", count=300, most=300000, pick=7),
        # Everything of a 7B model that is not projected, moments in 8 bits.
        _tensors("adamw_7b_q8", "adamw", "model", "bf16", "bf16", "q8", count=65, hidden=4096, vocab=32000),
        # The norm of the gains' gradients, and of everything's in a 7B model.
        _tensors("grad_norm_gains_7b", "grad_norm", "gains", "f32", "f32", count=65, hidden=4096),
        _tensors("grad_norm_7b", "grad_norm", "model", "bf16", "bf16", count=65, hidden=4096, vocab=32000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["forward", "backward", "backward", "adamw", "adamw", "grad_norm"])
    if kind in ("forward", "backward"):
        n = _log_int(rng, 64, 16384)
        if rng.random() < 0.66:
            n = n // 8 * 8
        T = _log_int(rng, 1, min(131072, MOST_ACTIVATIONS // n))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if dtype == "f32":
            T = max(1, T // 2)
        return _norm(None, kind, T, n, rng.choice(["layer", "rms"]), dtype, rng.choice(["f32", "bf16"]),
                     add=rng.random() < 0.5, bias=rng.random() < 0.5, serve=rng.random() < 0.3)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    gdtype = dtype if rng.random() < 0.6 else "f32"
    moments = rng.choice(["f32", "q8"]) if kind == "adamw" else None
    how = rng.choice(["gains", "model", "ragged", "ragged"])
    if how == "ragged":
        return _tensors(None, kind, how, dtype, gdtype, moments, count=_log_int(rng, 1, 400),
                        most=_log_int(rng, 10, 1000000), pick=rng.randrange(1 << 20))
    hidden = _log_int(rng, 256, 4096) // 128 * 128
    count = rng.randrange(5, 82, 2)
    if how == "gains":
        return _tensors(None, kind, how, dtype, gdtype, moments, count=count, hidden=hidden)
    vocab = _log_int(rng, 1000, min(128000, MOST_ELEMENTS // (4 * hidden)))
    return _tensors(None, kind, how, dtype, gdtype, moments, count=count, hidden=hidden, vocab=vocab)


def _sizes(case):
    if case["tensors"] == "gains":
        return [case["hidden"]] * case["count"]
    if case["tensors"] == "model":
        return [case["vocab"] * case["hidden"]] * 2 + [case["hidden"]] * case["count"]
    rng = random.Random(case["pick"])
    return [_log_int(rng, 1, case["most"]) for _ in range(case["count"])]


# ---------------------------------------------------------------------------------- inputs
def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000 + what)
    return g


def _normal(shape, dtype, scale, gen):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        b = min(flat.numel(), a + (1 << 26))
        flat[a:b] = torch.randn(b - a, generator=gen, device=DEV).mul_(scale)
    return out


def _activations(T, n, dtype, gen):
    """Rows of differing size and mean, a few features far larger than the rest."""
    out = torch.empty((T, n), dtype=dtype, device=DEV)
    feature = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.002, 20.0, 1.0)
    rows = max(1, (1 << 26) // n)
    for a in range(0, T, rows):
        k = min(rows, T - a)
        z = torch.randn((k, n), generator=gen, device=DEV).mul_(feature)
        z.add_(torch.randn((k, 1), generator=gen, device=DEV).mul_(0.3))
        out[a:a + k] = z.mul_(torch.exp(torch.randn((k, 1), generator=gen, device=DEV).mul_(0.5)))
    return out


def _prepare_norm(case, seed):
    T, n, dt, gdt = case["T"], case["n"], DTYPES[case["dtype"]], DTYPES[case["gdtype"]]
    s = {"case": case}
    s["gain"] = (1.0 + 0.1 * torch.randn(n, generator=_gen(seed, 1), device=DEV)).to(gdt)
    s["bias"] = (0.1 * torch.randn(n, generator=_gen(seed, 2), device=DEV)).to(gdt) if case["bias"] else None
    if case["kind"] == "forward":
        s["X"] = _activations(T, n, dt, _gen(seed, 3))
        s["R"] = _normal((T, n), dt, 0.5, _gen(seed, 4)) if case["add"] else None
        s["H"] = torch.empty((T, n), dtype=dt, device=DEV) if case["add"] else None
        s["Y"] = torch.empty((T, n), dtype=dt, device=DEV)
        keep = not case["serve"]
        s["mean"] = torch.empty(T, device=DEV) if keep and case["norm"] == "layer" else None
        s["rstd"] = torch.empty(T, device=DEV) if keep else None
        return s
    s["H"] = _activations(T, n, dt, _gen(seed, 3))
    s["dY"] = _normal((T, n), dt, 0.1, _gen(seed, 5))
    s["dR"] = _normal((T, n), dt, 0.1, _gen(seed, 6)) if case["add"] else None
    # what the forward pass kept
    rows = max(1, (1 << 26) // n)
    s["mean"] = torch.empty(T, device=DEV) if case["norm"] == "layer" else None
    s["rstd"] = torch.empty(T, device=DEV)
    for a in range(0, T, rows):
        h = s["H"][a:a + rows].double()
        if case["norm"] == "layer":
            mean = h.mean(1, keepdim=True)
            s["mean"][a:a + rows] = mean[:, 0]
            h -= mean
        s["rstd"][a:a + rows] = 1.0 / torch.sqrt(h.square().mean(1) + EPS_NORM)
    s["dX"] = torch.empty((T, n), dtype=dt, device=DEV)
    s["dgain"] = torch.empty(n, device=DEV)
    s["dbias"] = torch.empty(n, device=DEV) if case["bias"] else None
    if own:
        from paper_2406_17660_amd import grass
        s["ws"] = grass.workspace(grass.norm_backward_workspace(T, n, grass.F32 if case["dtype"] == "f32" else grass.BF16))
    return s


def _two_to(e):
    """2^e in fp32 from whole numbers e that it can hold."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _as_q8(values, top, dtype):
    """Codes and block scales of a state under way (rounded to the nearest code)."""
    scale = _two_to(torch.clamp(torch.frexp(values.abs().amax(1, keepdim=True))[1] - 1, min=-103) - top)
    return (values / scale).to(dtype), scale.view(-1).contiguous()


def _prepare_tensors(case, seed):
    sizes = _sizes(case)
    N = sum(sizes)
    wdt, gdt = DTYPES[case["dtype"]], DTYPES[case["gdtype"]]
    # Gradients of differing size from place to place; of an embedding most rows have none.
    G = _normal((N,), gdt, 0.01, _gen(seed, 1))
    if case["tensors"] == "model":
        V, h = case["vocab"], case["hidden"]
        some = (torch.rand((V, 1), generator=_gen(seed, 2), device=DEV) < 0.4).to(gdt)
        G[:V * h].view(V, h).mul_(some)
    s = {"case": case, "G": G}
    starts = [0]
    for k in sizes:
        starts.append(starts[-1] + k)
    parts = lambda flat: [flat[a:b] for a, b in zip(starts, starts[1:])]  # noqa: E731
    if case["kind"] == "grad_norm":
        s["out"] = torch.empty(2, device=DEV)
        if own:
            from paper_2406_17660_amd import grass
            s["plan"] = grass.adamw_plan(None, parts(G), None, None)
            s["ws"] = grass.workspace(grass.grad_norm_workspace(s["plan"]))
        return s
    s["W"] = _normal((N,), wdt, 0.02, _gen(seed, 3))
    # No decay of gains and other small tensors.
    decay = [0.0 if k < 65536 else 0.1 for k in sizes]
    s["decay"] = torch.repeat_interleave(torch.tensor(decay, device=DEV), torch.tensor(sizes, device=DEV), output_size=N)
    s["grad_scale"] = torch.tensor([GRAD_SCALE], device=DEV)
    s["t"] = ADAM_T
    s["M"] = _normal((N,), torch.float32, 0.001, _gen(seed, 4))
    s["V"] = torch.exp(_normal((N,), torch.float32, 1.0, _gen(seed, 5))).mul_(1e-5)
    if case["moments"] == "q8":
        # the elements of each block; where a tensor ends inside its last block, N for what is behind it
        s["blocks"] = None
        M, V = s["M"], s["V"]
        if case["tensors"] == "ragged":
            size = torch.tensor(sizes, device=DEV)
            count = (size + BLOCK - 1) // BLOCK
            nb = int(count.sum())
            tensor = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), count, output_size=nb)
            at = torch.arange(nb, device=DEV) - (count.cumsum(0) - count)[tensor]
            place = at.view(-1, 1) * BLOCK + torch.arange(BLOCK, device=DEV)
            start = torch.tensor(starts[:-1], device=DEV)[tensor].view(-1, 1)
            s["blocks"] = torch.where(place < size[tensor].view(-1, 1), start + place, N)
            zero = torch.zeros(1, device=DEV)
            M, V = torch.cat([M, zero])[s["blocks"]], torch.cat([V, zero])[s["blocks"]]
        M, s["mscale"] = _as_q8(M.view(-1, BLOCK), 7, torch.float8_e4m3fn)
        V, s["vscale"] = _as_q8(V.view(-1, BLOCK), 14, torch.float8_e5m2)
        if s["blocks"] is None:
            s["M"], s["V"] = M.view(-1), V.view(-1)
        else:
            inside = s["blocks"] < N
            s["M"] = M.view(torch.uint8)[inside].view(torch.float8_e4m3fn)
            s["V"] = V.view(torch.uint8)[inside].view(torch.float8_e5m2)
    if own:
        from paper_2406_17660_amd import grass
        scales = {}
        if case["moments"] == "q8":
            at = [0]
            for k in sizes:
                at.append(at[-1] + (k + BLOCK - 1) // BLOCK)
            scales = {name: [s[key][a:b] for a, b in zip(at, at[1:])] for name, key in (("Mscales", "mscale"), ("Vscales", "vscale"))}
        s["plan"] = grass.adamw_plan(parts(s["W"]), parts(G), parts(s["M"]), parts(s["V"]), weight_decay=decay, **scales)
    return s


def prepare(case, seed):
    return _prepare_norm(case, seed) if case["kind"] in ("forward", "backward") else _prepare_tensors(case, seed)


# ------------------------------------------------------------------------------ plain forms
def _plain_forward(s):
    rms = s["case"]["norm"] == "rms"
    h = s["X"].float()
    if s["R"] is not None:
        s["H"].copy_(h + s["R"].float())
        h = s["H"].float()
    mean = None if rms else h.mean(1, keepdim=True)
    d = h if rms else h - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS_NORM)
    y = d * rstd * s["gain"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    s["Y"].copy_(y)
    if s["rstd"] is not None:
        s["rstd"].copy_(rstd[:, 0])
        if not rms:
            s["mean"].copy_(mean[:, 0])


def _plain_backward(s):
    rms = s["case"]["norm"] == "rms"
    dy, d = s["dY"].float(), s["H"].float()
    rstd = s["rstd"].view(-1, 1)
    xhat = (d if rms else d - s["mean"].view(-1, 1)) * rstd
    s["dgain"].copy_((dy * xhat).sum(0))
    if s["dbias"] is not None:
        s["dbias"].copy_(dy.sum(0))
    z = dy * s["gain"].float()
    dx = z - xhat * (z * xhat).mean(1, keepdim=True)
    if not rms:
        dx = dx - z.mean(1, keepdim=True)
    dx = dx * rstd
    if s["dR"] is not None:
        dx = dx + s["dR"].float()
    s["dX"].copy_(dx)


def _f32(x):
    """A constant as fp32 has it."""
    return torch.tensor(x, dtype=torch.float32).item()


def _moments(s, g, m, v):
    """The new moments in fp32, every product and sum rounded by itself, and the update."""
    b1, b2 = _f32(BETA1), _f32(BETA2)
    m = m * b1 + g * _f32(1.0 - b1)
    v = v * b2 + (g * _f32(1.0 - b2)) * g
    c1, c2 = _f32(1.0 / (1.0 - b1 ** s["t"])), _f32(1.0 / (1.0 - b2 ** s["t"]))
    return m, v, _f32(LR) * (m * c1) / (torch.sqrt(v * c2) + _f32(EPS))


def _threshold(t, multiple, bits):
    """u of each place in a block at step t: the top bits of two whole numbers' products."""
    j = torch.arange(BLOCK, device=DEV, dtype=torch.int64)
    return (((j * 0x9E3779B1 + t * multiple) & 0xFFFFFFFF) >> (32 - bits)).double() / 2.0 ** bits


def _to_8_bits(x, u, top, low, step_bits, bits, dtype):
    """Blocks x (n x 128, fp32) as codes and scales.  In 64 bits: values next to a step's border."""
    fine = torch.isfinite(x)
    amax = torch.where(fine, x.abs(), 0.0).amax(1, keepdim=True)
    e = torch.clamp(torch.frexp(amax)[1] - 1, min=-103)
    e = torch.where(amax == 0, -103, e)
    scale = _two_to(e - top)
    a = torch.where(fine, x.abs(), 0.0).double() / scale.double()
    step = _two_to(torch.clamp(torch.frexp(a)[1] - 1, min=low) - step_bits).double()
    q = torch.floor(torch.round(a / step * 2.0 ** bits) / 2.0 ** bits + u) * step
    q = torch.where(fine, torch.where(torch.signbit(x), -q, q), math.nan)
    return q.float().to(dtype), scale.view(-1)


def _plain_adamw(s):
    g, w = s["G"].float() * s["grad_scale"], s["W"].float()
    if s["case"]["moments"] == "f32":
        s["M"][:], s["V"][:], u = _moments(s, g, s["M"], s["V"])
        s["W"].copy_(w * (1.0 - _f32(LR) * s["decay"]) - u)
        return
    at, M, V = s["blocks"], s["M"].float(), s["V"].float()
    if at is None:
        m, v = M.view(-1, BLOCK), V.view(-1, BLOCK)
        gb = g.view(-1, BLOCK)
    else:  # tensors that end inside a block: zeros behind their ends
        zero = torch.zeros(1, device=DEV)
        m, v, gb = (torch.cat([x, zero])[at] for x in (M, V, g))
    m, v, u = _moments(s, gb, m * s["mscale"].view(-1, 1), v * s["vscale"].view(-1, 1))
    qm, s["mscale"][:] = _to_8_bits(m, _threshold(s["t"], 0x6A09E667, 20), 7, -6, 3, 20, torch.float8_e4m3fn)
    qv, s["vscale"][:] = _to_8_bits(v, _threshold(s["t"], 0xBB67AE85, 21), 14, -14, 2, 21, torch.float8_e5m2)
    if at is None:
        s["M"].copy_(qm.view(-1))
        s["V"].copy_(qv.view(-1))
        u = u.view(-1)
    else:
        inside = at < g.numel()
        s["M"].view(torch.uint8).copy_(qm.view(torch.uint8)[inside])
        s["V"].view(torch.uint8).copy_(qv.view(torch.uint8)[inside])
        u = u[inside]
    s["W"].copy_(w * (1.0 - _f32(LR) * s["decay"]) - u)


def _plain_grad_norm(s):
    # in 64 bits: a long sum
    norm = torch.sqrt(s["G"].double().square().sum())
    s["out"][0] = norm
    s["out"][1] = torch.clamp(MAX_NORM / norm, max=1.0)


# ------------------------------------------------------------------------- the framework's
def _own(s):
    from paper_2406_17660_amd import grass
    case = s["case"]
    if case["kind"] == "adamw":
        grass.adamw_step(s["plan"], LR, BETA1, BETA2, EPS, s["t"], grad_scale=s["grad_scale"])
        return
    if case["kind"] == "grad_norm":
        grass.grad_norm(s["plan"], MAX_NORM, s["out"], s["ws"])
        return
    kind = grass.NORM_RMS if case["norm"] == "rms" else grass.NORM_LAYER
    if case["kind"] == "forward":
        grass.norm_forward(s["X"], s["gain"], s["bias"], EPS_NORM, s["Y"], kind, R=s["R"], H=s["H"], mean=s["mean"], rstd=s["rstd"])
    else:
        grass.norm_backward(s["dY"], s["H"], s["gain"], s["mean"], s["rstd"], s["dX"], s["dgain"], s["dbias"], s["ws"], kind, dR=s["dR"])


OUTPUTS = {"forward": ("H", "Y", "mean", "rstd"), "backward": ("dX", "dgain", "dbias"),
           "adamw": ("W", "M", "V", "mscale", "vscale"), "grad_norm": ("out",)}


def _outputs(s):
    return {k: s[k] for k in OUTPUTS[s["case"]["kind"]] if s.get(k) is not None}


def run(s):
    if own:
        _own(s)
    else:
        {"forward": _plain_forward, "backward": _plain_backward, "adamw": _plain_adamw,
         "grad_norm": _plain_grad_norm}[s["case"]["kind"]](s)
    return _outputs(s)


# ------------------------------------------------------------------------------------ work
def work(case):
    if case["kind"] in ("forward", "backward"):
        T, n, a = case["T"], case["n"], SIZE[case["dtype"]]
        arrays = 2 + (2 if case["add"] else 0) if case["kind"] == "forward" else 3 + case["add"]
        stats = 0 if case.get("serve") else (2 if case["norm"] == "layer" else 1)
        vectors = (1 + case["bias"]) * SIZE[case["gdtype"]]
        if case["kind"] == "backward":
            vectors = SIZE[case["gdtype"]] + (1 + case["bias"]) * 4
        return {"bytes": T * n * a * arrays + 4 * T * stats + n * vectors, "flops": T * n * (8 if case["kind"] == "forward" else 14)}
    sizes = _sizes(case)
    N = sum(sizes)
    if case["kind"] == "grad_norm":
        return {"bytes": N * SIZE[case["gdtype"]], "flops": 2 * N}
    each = SIZE[case["gdtype"]] + 2 * SIZE[case["dtype"]]
    if case["moments"] == "f32":
        return {"bytes": N * (each + 16), "flops": 16 * N}
    return {"bytes": N * (each + 4) + 16 * sum((k + BLOCK - 1) // BLOCK for k in sizes), "flops": 30 * N}


# ----------------------------------------------------------------------------------- exact
def _exact_norm(case, s):
    out = {k: torch.empty(s[k].shape, dtype=torch.float64, device=DEV) for k in OUTPUTS[case["kind"]]
           if s.get(k) is not None and k not in ("dgain", "dbias")}
    n, gain = case["n"], s["gain"].double()
    sums = torch.zeros((2, n), dtype=torch.float64, device=DEV)
    rows = max(1, (1 << 25) // n)
    for a in range(0, case["T"], rows):
        at = slice(a, a + rows)
        if case["kind"] == "forward":
            h = s["X"][at].double()
            if case["add"]:
                h = (h + s["R"][at].double()).to(DTYPES[case["dtype"]]).double()  # the sum that is stored is what is normed
                out["H"][at] = h
            mean = h.sum(1) / n if case["norm"] == "layer" else torch.zeros_like(h[:, 0])
            h -= mean[:, None]
            var = torch.linalg.vector_norm(h, dim=1) ** 2 / n
            y = h * (var + EPS_NORM)[:, None] ** -0.5 * gain
            out["Y"][at] = y + s["bias"].double() if case["bias"] else y
            if "rstd" in out:
                out["rstd"][at] = (var + EPS_NORM) ** -0.5
            if "mean" in out:
                out["mean"][at] = mean
            continue
        # the chain rule through y = gain * z / sigma + bias, z = h - mean(h), sigma = sqrt(mean(z^2) + eps)
        dy, z, inv = s["dY"][at].double(), s["H"][at].double(), s["rstd"][at].double()[:, None]
        if case["norm"] == "layer":
            z = z - s["mean"][at].double()[:, None]
        sums[0] += torch.einsum("tn,tn->n", dy, z * inv)
        sums[1] += torch.einsum("tn->n", dy)
        dz = dy * gain * inv
        dsigma = -(dy * gain * z).sum(1, keepdim=True) * inv ** 2
        dz += dsigma * z * inv / n
        if case["norm"] == "layer":
            # z's mean is zero but for the rounding of the kept mean, so only dy's part has one
            dz -= (dy * gain * inv).mean(1, keepdim=True)
        out["dX"][at] = dz + s["dR"][at].double() if case["add"] else dz
    if case["kind"] == "backward":
        out["dgain"] = sums[0]
        if case["bias"]:
            out["dbias"] = sums[1]
    return out


def _exact_q8(x, tensor_block, nblocks, place, t, multiple, top, low, man):
    """x (fp64 values of fp32 numbers, flat) in blocks numbered by `tensor_block`: code values and scales."""
    def binade(y, least):  # the power of two at or below y: its exponent field alone
        return (torch.clamp(y, min=2.0 ** least).view(torch.int64) >> 52 << 52).view(torch.float64)

    amax = torch.zeros(nblocks, dtype=torch.float64, device=DEV).scatter_reduce_(0, tensor_block, x.abs(), "amax")
    scale = binade(amax, -103) * 2.0 ** -top
    a = x / scale[tensor_block]
    step = binade(a.abs(), low) * 2.0 ** -man
    fraction = 2.0 ** (23 - man)
    u = torch.floor(torch.remainder(place.double() * 0x9E3779B1 + float(t * multiple % 2 ** 32), 2.0 ** 32) / 2.0 ** (9 + man)) / fraction
    whole = torch.floor(torch.round(a.abs() / step * fraction) / fraction + u)
    return torch.sign(x) * whole * step, scale


def _exact_adamw(case, s):
    sizes = _sizes(case)
    q8 = case["moments"] == "q8"

    def r32(x):  # the values that are then cut to 8 bits are fp32's: a product or sum of two fp32 numbers as fp32 rounds it
        return x.float().double() if q8 else x

    N = sum(sizes)
    b1, b2, lr, eps = (float(torch.tensor(x, dtype=torch.float32)) for x in (BETA1, BETA2, LR, EPS))
    t = s["t"]
    out = {}
    g = r32(s["G"].double() * s["grad_scale"].double())
    m, v = s["M"].to(torch.float32).double(), s["V"].to(torch.float32).double()
    if q8:
        size = torch.tensor(sizes, device=DEV)
        count = (size + BLOCK - 1) // BLOCK
        which = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), size, output_size=N)
        inside = torch.arange(N, device=DEV) - (size.cumsum(0) - size)[which]
        block = (count.cumsum(0) - count)[which] + inside // BLOCK
        place = inside % BLOCK
        del which, inside
        m *= s["mscale"].double()[block]
        v *= s["vscale"].double()[block]
    m = r32(r32(b1 * m) + r32(float(torch.tensor(1 - b1, dtype=torch.float32)) * g))
    v = r32(r32(b2 * v) + r32(r32(float(torch.tensor(1 - b2, dtype=torch.float32)) * g) * g))
    step = lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    out["W"] = s["W"].double() * (1 - lr * s["decay"].double()) - step
    del g, step
    if not q8:
        return {**out, "M": m, "V": v}
    nb = int(count.sum())
    out["M"], out["mscale"] = _exact_q8(m, block, nb, place, t, 0x6A09E667, 7, -6, 3)
    del m
    out["V"], out["vscale"] = _exact_q8(v, block, nb, place, t, 0xBB67AE85, 14, -14, 2)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("forward", "backward"):
        return _exact_norm(case, s)
    if case["kind"] == "grad_norm":
        norm = torch.linalg.vector_norm(s["G"].double())
        return {"out": torch.stack([norm, (MAX_NORM / norm).clamp(max=1.0)])}
    return _exact_adamw(case, s)
