"""The operators at the two ends of a model, as timed cases: the embedding lookup and its gradient by
tokens, and the log probabilities of given tokens with entropy and top alternatives, and their gradient.

A case is a dict of plain values:

  kind      "embed_forward", "embed_backward", "logp_forward" or "logp_backward"
  T, V      tokens and vocabulary
  n         features of an embedding
  dtype     type of the embedding (its gradient in "embed_backward"), or of the logits and their gradient
  adtype    type of the rows that an embedding gives (of their gradient in "embed_backward")
  itype     type of the token numbers, "i32" or "i64"
  scaled    embedding: rows are multiplied by sqrt(n); logits: by 0.7, the inverse of a temperature
  tokens    "zipf": as often as in text; "uniform": each as often as any other
  padded    every tenth token is padding (-1 among the tokens, -100 among the targets)
  add       embed_backward: added to what is there (a head that shares the embedding has left its gradient)
  top       logp_forward: the number of alternatives that are asked for
  entropy   the entropies are asked for, or have a gradient
  keep      logp_forward: what the backward pass needs is kept
  masked    some rows allow eight tokens, one in 64 allows none: the others' logits are minus infinity
  off       elements by which rows of logits are apart beyond V, and by which the first is off the start

The gradient of a row of an embedding is the sum over the places where its token stands; tokens outside the
vocabulary have rows of zeros and give no gradient.  Targets outside the vocabulary have log
probability 0 and give no gradient.  A row of logits that are all minus infinity has log probabilities of
minus infinity, entropy 0 and no gradient.  Alternatives are in falling order of the logits, ties by the
lower token; where fewer have a probability the rest is token -1 with log probability minus infinity.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ITYPES = {"i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
INVERSE_TEMPERATURE = 0.7
ALLOWED = 8
MOST_FEATURES = 131072 * 4096  # a drawn case stays under the largest listed ones
MOST_WEIGHTS = 32000 * 4096
MOST_LOGITS = 32768 * 32000
MOST_RANKED = 256 * 128000  # of cases with alternatives, whose plain form sorts


def _embed(name, kind, T, V, n, dtype, adtype, itype="i64", scaled=False, tokens="zipf", padded=False, add=False):
    case = {"kind": kind, "T": T, "V": V, "n": n, "dtype": dtype, "adtype": adtype, "itype": itype, "scaled": scaled,
            "tokens": tokens, "padded": padded}
    if kind == "embed_backward":
        case["add"] = add
    return {"name": name, **case} if name else case


def _logp(name, kind, T, V, dtype, itype="i64", scaled=False, padded=False, top=0, entropy=False, keep=False, masked=False, off=0):
    case = {"kind": kind, "T": T, "V": V, "dtype": dtype, "itype": itype, "scaled": scaled, "padded": padded,
            "entropy": entropy, "masked": masked, "off": off}
    if kind == "logp_forward":
        case.update(top=top, keep=keep)
    return {"name": name, **case} if name else case


def listed():
    return [
        # The next token of eight texts, as they are written: latency.
        _embed("embed_token", "embed_forward", 8, 32000, 4096, "bf16", "bf16"),
        # A 7B model's full token batch.
        _embed("embed_7b", "embed_forward", 131072, 32000, 4096, "bf16", "bf16"),
        # fp32 weights, an odd width, padded texts of any length, rows scaled as where embedding and head are one.
        _embed("embed_odd", "embed_forward", 2407, 10007, 1293, "f32", "bf16", itype="i32", scaled=True, padded=True),
        # The smallest model's embedding in training.
        _embed("embed_grad_60m", "embed_backward", 65536, 32000, 512, "f32", "bf16"),
        # A 7B model's embedding over the full token batch.
        _embed("embed_grad_7b", "embed_backward", 131072, 32000, 4096, "bf16", "bf16"),
        # A short padded batch in fine-tuning at the 1B model's odd inner width, added to the gradient of a head that shares the weights.
        _embed("embed_grad_odd", "embed_backward", 2047, 32000, 5461, "f32", "bf16", itype="i32", scaled=True, padded=True, add=True),
        # One text's next token with its alternatives, as it is written: latency.
        _logp("logp_token", "logp_forward", 1, 32000, "bf16", scaled=True, top=20, entropy=True),
        # The loss of a long batch, with what its gradient needs.
        _logp("logp_7b", "logp_forward", 32768, 32000, "bf16", padded=True, keep=True),
        # The next tokens of many texts from a large vocabulary, some of them bound to a grammar.
        _logp("logp_serve", "logp_forward", 256, 128000, "f32", itype="i32", scaled=True, top=20, entropy=True, masked=True),
        # Scoring texts under an odd vocabulary, rows of logits cut out of larger ones.
        _logp("logp_odd", "logp_forward", 1025, 50001, "bf16", top=5, entropy=True, padded=True, off=7),
        # The loss's gradient over a long batch.
        _logp("logp_grad_7b", "logp_backward", 32768, 32000, "bf16", padded=True),
        # A policy's gradient with an entropy bonus, odd vocabulary.
        _logp("logp_grad_odd", "logp_backward", 513, 50001, "f32", scaled=True, entropy=True, masked=True, off=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed_forward", "embed_backward", "embed_backward", "logp_forward", "logp_forward", "logp_backward"])
    dtype, itype = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["i32", "i64", "i64"])
    scaled, padded = rng.random() < 0.4, rng.random() < 0.4
    if kind.startswith("embed"):
        n = _log_int(rng, 16, 16384)
        if rng.random() < 0.66:
            n = n // 8 * 8
        V = _log_int(rng, 50, min(256000, MOST_WEIGHTS // n))
        T = _log_int(rng, 1, min(131072, MOST_FEATURES // n))
        adtype = dtype if rng.random() < 0.5 else rng.choice(["bf16", "f32"])
        if "f32" in (dtype, adtype):
            T, V = max(1, T // 2), max(25, V // 2)
        return _embed(None, kind, T, V, n, dtype, adtype, itype, scaled, rng.choice(["zipf", "zipf", "uniform"]), padded,
                      add=rng.random() < 0.4)
    V = _log_int(rng, 2, 256000)
    if rng.random() < 0.5:
        V = (V + 7) // 8 * 8
    top = min(V, _log_int(rng, 1, 64)) if kind == "logp_forward" and rng.random() < 0.5 else 0
    T = _log_int(rng, 1, min(32768, (MOST_RANKED if top else MOST_LOGITS // 2 if dtype == "f32" else MOST_LOGITS) // V))
    return _logp(None, kind, T, V, dtype, itype, scaled, padded, top=top, entropy=rng.random() < 0.4, keep=rng.random() < 0.6,
                 masked=rng.random() < 0.3, off=rng.choice([0, 0, 0, 8, rng.randrange(1, 16)]))


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


def _tokens(T, V, how, seed):
    """T token numbers; by Zipf's law the k-th most frequent one is as likely as 1 / (k + 2.7)."""
    u = torch.rand(T, generator=_gen(seed, 1), device=DEV, dtype=torch.float64)
    if how == "uniform":
        return (u * V).long().clamp(max=V - 1)
    weight = (1.0 / (torch.arange(V, device=DEV, dtype=torch.float64) + 2.7)).cumsum(0)
    rank = torch.searchsorted(weight, u * weight[-1]).clamp(max=V - 1)
    return torch.randperm(V, generator=_gen(seed, 2), device=DEV)[rank]


def _with_padding(ids, case, seed, value):
    if case["padded"]:
        ids = torch.where(torch.rand(ids.numel(), generator=_gen(seed, 3), device=DEV) < 0.1, value, ids)
    return ids.to(ITYPES[case["itype"]])


def _prepare_embed(case, seed):
    T, V, n = case["T"], case["V"], case["n"]
    s = {"case": case, "scale": math.sqrt(n) if case["scaled"] else 1.0}
    s["ids"] = _with_padding(_tokens(T, V, case["tokens"], seed), case, seed, -1)
    if case["kind"] == "embed_forward":
        s["E"] = _normal((V, n), DTYPES[case["dtype"]], 0.02, _gen(seed, 4))
        s["Y"] = torch.empty((T, n), dtype=DTYPES[case["adtype"]], device=DEV)
        return s
    s["dY"] = _normal((T, n), DTYPES[case["adtype"]], 0.01, _gen(seed, 5))
    if case["add"]:
        s["dE"] = _normal((V, n), DTYPES[case["dtype"]], 0.01, _gen(seed, 6))
    else:
        s["dE"] = torch.empty((V, n), dtype=DTYPES[case["dtype"]], device=DEV)
    if own:
        from paper_2406_17660_amd import grass
        s["ws"] = grass.workspace(grass.embed_backward_workspace(T, V, n))
    return s


def _rows_of(case):
    """Slices of rows that are worked on at a time where inputs are made and in 64 bits."""
    rows = max(1, (1 << 26) // case["V"])
    return [slice(a, min(a + rows, case["T"])) for a in range(0, case["T"], rows)]


def _logits(case, targets, seed):
    """Logits of a language model: frequent tokens higher than rare ones, and the right one mostly well above
    the others; rows cut out of longer ones where the case says so."""
    T, V, off = case["T"], case["V"], case["off"]
    out = torch.empty(off + T * (V + off), dtype=DTYPES[case["dtype"]], device=DEV)[off:].view(T, V + off)[:, :V]
    unigram = -torch.log(torch.randperm(V, generator=_gen(seed, 2), device=DEV).float() + 2.7)
    gen, height = _gen(seed, 4), torch.randn((T, 1), generator=_gen(seed, 5), device=DEV).mul_(3.0).add_(8.0)
    how = torch.rand((T, 1), generator=_gen(seed, 6), device=DEV)
    row = torch.arange(T, device=DEV).view(-1, 1)
    for at in _rows_of(case):
        z = torch.randn((at.stop - at.start, V), generator=gen, device=DEV).mul_(2.0).add_(unigram)
        z.scatter_add_(1, targets[at].view(-1, 1), height[at])
        if case["masked"]:
            allowed = torch.randint(V, (z.shape[0], ALLOWED), generator=gen, device=DEV)
            some = torch.zeros_like(z, dtype=torch.bool).scatter_(1, allowed, True)
            some.scatter_(1, targets[at].view(-1, 1), True)
            z = torch.where(some | (how[at] > 0.25), z, -math.inf)
            z = torch.where(row[at] % 64 == 3, -math.inf, z)
        out[at] = z
    return out


def _prepare_logp(case, seed):
    T, V, dt = case["T"], case["V"], DTYPES[case["dtype"]]
    s = {"case": case, "scale": INVERSE_TEMPERATURE if case["scaled"] else 1.0}
    targets = _tokens(T, V, "zipf", seed)
    s["logits"] = _logits(case, targets, seed)
    s["targets"] = _with_padding(targets, case, seed, -100)
    f32 = {"dtype": torch.float32, "device": DEV}
    if case["kind"] == "logp_forward":
        s["logp"] = torch.empty(T, **f32)
        s["entropy"] = torch.empty(T, **f32) if case["entropy"] else None
        s["rmax"], s["rlog"] = (torch.empty(T, **f32) if case["keep"] else None for _ in range(2))
        k = case["top"]
        s["top_logp"] = torch.empty((T, k), **f32) if k else None
        s["top_idx"] = torch.empty((T, k), dtype=torch.int32, device=DEV) if k else None
        if own:
            from paper_2406_17660_amd import grass
            s["ws"] = grass.workspace(grass.logp_forward_workspace(T, V, k, grass.F32 if case["dtype"] == "f32" else grass.BF16))
        return s
    # what the forward pass kept
    s["rmax"], s["rlog"] = torch.empty(T, **f32), torch.empty(T, **f32)
    s["entropy"] = torch.empty(T, **f32) if case["entropy"] else None
    for at in _rows_of(case):
        x = s["logits"][at].double()
        m = x.amax(1, keepdim=True)
        none = m == -math.inf
        d = (x - torch.where(none, 0.0, m)) * s["scale"]
        total = d.exp().sum(1, keepdim=True)
        log = torch.where(none, 0.0, total.log())
        s["rmax"][at], s["rlog"][at] = m[:, 0], log[:, 0]
        if case["entropy"]:
            e = (d.exp() * torch.where(d == -math.inf, 0.0, d)).sum(1, keepdim=True)
            s["entropy"][at] = torch.where(none, 0.0, log - e / total)[:, 0]
    # of a mean over the tokens, weighted as by advantages where there is an entropy bonus
    weight = torch.randn(T, generator=_gen(seed, 7), device=DEV) if case["entropy"] else torch.ones(T, device=DEV)
    s["dlogp"] = weight.mul_(-1.0 / T)
    s["dentropy"] = torch.full((T,), -0.01 / T, device=DEV) if case["entropy"] else None
    s["dlogits"] = torch.empty((T, V), dtype=dt, device=DEV)
    return s


def prepare(case, seed):
    return _prepare_embed(case, seed) if case["kind"].startswith("embed") else _prepare_logp(case, seed)


# ------------------------------------------------------------------------------ plain forms
def _plain_embed_forward(s):
    V = s["E"].shape[0]
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < V)
    y = s["E"][torch.where(there, ids, 0)].float() * s["scale"]
    s["Y"].copy_(torch.where(there.view(-1, 1), y, 0.0))


def _plain_embed_backward(s):
    V, n = s["dE"].shape
    ids = s["ids"].long()
    # (a row behind the last for what is no token)
    ids = torch.where((ids >= 0) & (ids < V), ids, V)
    total = torch.zeros((V + 1, n), device=DEV).index_add_(0, ids, s["dY"].float())[:V] * s["scale"]
    s["dE"].copy_(s["dE"].float() + total if s["case"]["add"] else total)


def _shifted(s):
    """The logits and their rows' largest, the rows without any, and the scaled differences."""
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    none = m == -math.inf
    return x, m, none, (x - torch.where(none, 0.0, m)) * s["scale"]


def _plain_logp_forward(s):
    x, m, none, d = _shifted(s)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log = torch.where(none, 0.0, total.log())
    targets = s["targets"].long().view(-1, 1)
    there = (targets >= 0) & (targets < x.shape[1])
    logp = d.gather(1, torch.where(there, targets, 0)) - log
    s["logp"].copy_(torch.where(there, logp, 0.0)[:, 0])
    if s["entropy"] is not None:
        mean = (e * torch.where(d == -math.inf, 0.0, d)).sum(1, keepdim=True) / total
        s["entropy"].copy_(torch.where(none, 0.0, log - mean)[:, 0])
    if s["rmax"] is not None:
        s["rmax"].copy_(m[:, 0])
        s["rlog"].copy_(log[:, 0])
    if s["top_idx"] is not None:
        # whole numbers in the order of the logits, then of the tokens: no two alike
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        order = order * (1 << 32) - torch.arange(x.shape[1], device=DEV)
        at = torch.topk(order, s["top_idx"].shape[1], dim=1).indices
        top = d.gather(1, at) - log
        s["top_logp"].copy_(top)
        s["top_idx"].copy_(torch.where(top == -math.inf, -1, at))


def _plain_logp_backward(s):
    x = s["logits"].float()
    m, log = s["rmax"].view(-1, 1), s["rlog"].view(-1, 1)
    logp = (x - torch.where(m == -math.inf, 0.0, m)) * s["scale"] - log
    p = logp.exp()
    targets = s["targets"].long().view(-1, 1)
    there = (targets >= 0) & (targets < x.shape[1]) & (m > -math.inf)
    dlogp = torch.where(there, s["dlogp"].view(-1, 1), 0.0)
    dx = -dlogp * p
    dx.scatter_add_(1, torch.where(there, targets, 0), dlogp)
    if s["dentropy"] is not None:
        dx = dx - s["dentropy"].view(-1, 1) * p * (torch.where(logp == -math.inf, 0.0, logp) + s["entropy"].view(-1, 1))
    s["dlogits"].copy_(dx * s["scale"])


# ------------------------------------------------------------------------- the framework's
def _own(s):
    from paper_2406_17660_amd import grass
    kind = s["case"]["kind"]
    if kind == "embed_forward":
        grass.embed_forward(s["E"], s["ids"], s["Y"], s["scale"])
    elif kind == "embed_backward":
        grass.embed_backward(s["dY"], s["ids"], s["dE"], s["ws"], s["scale"], accumulate=s["case"]["add"])
    elif kind == "logp_forward":
        grass.logp_forward(s["logits"], s["targets"], s["logp"], s["ws"], s["scale"], entropy=s["entropy"], rmax=s["rmax"],
                           rlog=s["rlog"], top_logp=s["top_logp"], top_idx=s["top_idx"])
    else:
        grass.logp_backward(s["logits"], s["targets"], s["rmax"], s["rlog"], s["dlogp"], s["dlogits"], s["scale"],
                            entropy=s["entropy"], dentropy=s["dentropy"])


OUTPUTS = {"embed_forward": ("Y",), "embed_backward": ("dE",),
           "logp_forward": ("logp", "entropy", "rmax", "rlog", "top_logp", "top_idx"), "logp_backward": ("dlogits",)}


def _outputs(s):
    return {k: s[k] for k in OUTPUTS[s["case"]["kind"]] if s.get(k) is not None}


def run(s):
    if own:
        _own(s)
    else:
        {"embed_forward": _plain_embed_forward, "embed_backward": _plain_embed_backward,
         "logp_forward": _plain_logp_forward, "logp_backward": _plain_logp_backward}[s["case"]["kind"]](s)
    return _outputs(s)


# ------------------------------------------------------------------------------------ work
def work(case):
    T, V, index = case["T"], case["V"], SIZE[case["itype"]]
    if case["kind"].startswith("embed"):
        n, weights, rows = case["n"], SIZE[case["dtype"]], SIZE[case["adtype"]]
        touched = min(T, V)  # rows of the embedding that are read or added to, at the most
        if case["kind"] == "embed_forward":
            return {"bytes": T * (index + n * rows) + touched * n * weights, "flops": T * n}
        there = 2 * touched if case["add"] else V
        return {"bytes": T * (index + n * rows) + there * n * weights, "flops": T * n + touched * n}
    logits = T * V * SIZE[case["dtype"]]
    if case["kind"] == "logp_backward":
        return {"bytes": 2 * logits + T * (index + 12 + 8 * case["entropy"]), "flops": T * V * (8 if case["entropy"] else 5)}
    return {"bytes": logits + T * (index + 4 + 4 * case["entropy"] + 8 * case["keep"] + 8 * case["top"]),
            "flops": T * V * (7 if case["entropy"] else 5)}


# ----------------------------------------------------------------------------------- exact
def _exact_embed(case, s):
    ids = s["ids"].double()
    where = torch.nonzero((ids >= 0) & (ids <= case["V"] - 1))[:, 0]
    ids = s["ids"][where].to(torch.int64)
    if case["kind"] == "embed_forward":
        out = torch.zeros(s["Y"].shape, dtype=torch.float64, device=DEV)
        for a in range(0, where.numel(), 16384):
            out[where[a:a + 16384]] = torch.index_select(s["E"], 0, ids[a:a + 16384]).double() * s["scale"]
        return {"Y": out}
    out = s["dE"].double() if case["add"] else torch.zeros(s["dE"].shape, dtype=torch.float64, device=DEV)
    # the same places of a token one behind the other: differences of running sums would lose digits, so rows are added by scattering
    columns = max(1, (1 << 27) // max(1, case["T"]))
    for a in range(0, case["n"], columns):
        part = s["dY"][:, a:a + columns][where].double() * s["scale"]
        out[:, a:a + columns] = out[:, a:a + columns].contiguous().scatter_add_(0, ids.view(-1, 1).expand(-1, part.shape[1]), part)
    return {"dE": out}


def _exact_logp_forward(case, s):
    T, k = case["T"], case["top"]
    out = {name: torch.empty(s[name].shape, dtype=torch.float64, device=DEV) for name in OUTPUTS["logp_forward"]
           if s.get(name) is not None and name != "top_idx"}
    for at in _rows_of(case):
        z = s["logits"][at].double()
        top = z.max(1).values
        z *= s["scale"]
        empty = torch.isneginf(top)
        lse = torch.logsumexp(z, 1)
        logp = torch.where(empty[:, None], -math.inf, z - lse[:, None])
        target = s["targets"][at].to(torch.int64)
        right = torch.zeros(target.shape, dtype=torch.float64, device=DEV)
        for_real = torch.nonzero((0 <= target) & (target < case["V"]))[:, 0]
        right[for_real] = logp[for_real, target[for_real]]
        out["logp"][at] = right
        if case["entropy"]:
            out["entropy"][at] = torch.special.entr(logp.exp()).sum(1)
        if case["keep"]:
            out["rmax"][at] = top
            out["rlog"][at] = torch.where(empty, 0.0, lse - top * s["scale"])
        if k:
            out["top_logp"][at] = torch.sort(logp, dim=1, descending=True).values[:, :k]
    return {**out, "top_idx": None} if k else out


def _exact_logp_backward(case, s):
    out = torch.empty(s["dlogits"].shape, dtype=torch.float64, device=DEV)
    for at in _rows_of(case):
        lse = s["rmax"][at].double() * s["scale"] + s["rlog"][at].double()
        some = torch.isfinite(lse)
        logp = s["logits"][at].double() * s["scale"] - torch.where(some, lse, 0.0)[:, None]
        p = torch.exp(logp)
        target = s["targets"][at].to(torch.int64)
        counted = torch.nonzero((target >= 0) & (target < case["V"]) & some)[:, 0]
        # d logp_target = onehot - p, d H = -p (log p + H), through z = scale x
        dz = torch.zeros_like(p)
        dz[counted] = -p[counted] * s["dlogp"][at].double()[counted, None]
        dz[counted, target[counted]] += s["dlogp"][at].double()[counted]
        if case["entropy"]:
            plogp = -torch.special.entr(p)
            dz -= (plogp + p * s["entropy"][at].double()[:, None]) * s["dentropy"][at].double()[:, None]
        out[at] = dz * s["scale"]
    return {"dlogits": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("embed"):
        return _exact_embed(case, s)
    return _exact_logp_forward(case, s) if case["kind"] == "logp_forward" else _exact_logp_backward(case, s)
