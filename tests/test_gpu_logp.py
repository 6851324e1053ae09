"""grass_logp_forward and grass_logp_backward against the same formulas in 64 bits.

Tolerances, in half steps of fp32, U = 2^-24.  With d = scale * (x - rmax): the difference and the product are
rounded once each, and d is turned into a power of two, so that an exponential is off by (3 |d| + 4) U of itself.
The sum of exponentials has at most 256 values one behind the other (a thread's, then trees over threads and parts), so
that it is off by (256 + 3 E + 4) U of itself, where E, the mean of |d| over the distribution, is entropy - rlog (the
entropy is the mean of -log p = rlog - d, and d = -|d|); rlog is the logarithm of that, rounded: SUM = 264 + 3 E + rlog.  log p is off by SUM + 4 (|d| + |rlog|); the entropy,
rlog - (sum of exponentials times d) / (their sum), by SUM (1 + E) + 4 (rlog + E).  In the backward pass, where rmax and rlog are
given, p is off by (4 (|d| + rlog) + 8) U of itself."""
import numpy as np
import pytest
import torch

import ends_ref
from gpu_util import DEV, to_f64
from paper_2406_17660_amd import grass

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
TINY = 2.0 ** -120  # what is below the normal numbers may be zero
INF, NAN = float("inf"), float("nan")


def draw(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def whole(shape, seed, most):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(most, shape, generator=g, device=DEV)


def nan(shape, dtype=F32):
    return torch.full(shape, NAN, dtype=dtype, device=DEV)


def code(dtype):
    return grass.F32 if dtype == F32 else grass.BF16


def padded(t, ld, offset):
    """The values of t in rows ld elements apart, the first `offset` elements behind the base; plus infinity around them."""
    T, n = t.shape
    flat = torch.full((offset + T * ld + 8,), INF, dtype=t.dtype, device=DEV)
    view = flat[offset:offset + T * ld].view(T, ld)[:, :n]
    view.copy_(t)
    return view, flat


def forward(x, targets, top, scale=1.0, entropy=True, keep=True):
    T, V = x.shape
    out = {"logp": nan((T,)) if targets is not None else None, "entropy": nan((T,)) if entropy else None,
           "rmax": nan((T,)) if keep else None, "rlog": nan((T,)) if keep else None, "top_logp": nan((T, top)) if top else None,
           "top_idx": torch.full((T, top), -7, dtype=torch.int32, device=DEV) if top else None}
    need = grass.logp_forward_workspace(T, V, top, code(x.dtype))
    room = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    grass.logp_forward(x, targets, out["logp"], room[:need] if need else None, scale, entropy=out["entropy"], rmax=out["rmax"],
                       rlog=out["rlog"], top_logp=out["top_logp"], top_idx=out["top_idx"])
    assert bool((room[need:] == 0xFF).all()), "nothing behind the workspace is written"
    return out


def near(got, want, off):
    got = to_f64(got)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(all="ignore"):
        return (same | (np.abs(got - want) <= off)).all()


def check_forward(x, targets, scale, out):
    z = to_f64(x)
    m, rlog, logp, H = ends_ref.logp_rows(z, scale)
    E = H - rlog
    SUM = (264 + 3 * E + rlog) * U
    with np.errstate(all="ignore"):
        off = SUM[:, None] + 4 * U * (np.abs(logp + rlog[:, None]) + np.abs(rlog)[:, None])
    if out["rmax"] is not None:
        spoiled = np.isnan(rlog)
        assert np.array_equal(to_f64(out["rmax"])[~spoiled], m[~spoiled])
        assert near(out["rlog"], rlog, SUM)
    if out["entropy"] is not None:
        assert near(out["entropy"], H, SUM * (1 + E) + 4 * U * (rlog + E))
    if targets is not None:
        ids = targets.cpu().numpy().astype(np.int64)
        assert near(out["logp"], ends_ref.given(logp, ids), ends_ref.given(off, ids))
    if out["top_idx"] is not None:
        idx, val = ends_ref.alternatives(z, logp, out["top_idx"].shape[1])
        assert np.array_equal(out["top_idx"].cpu().numpy(), idx)
        assert near(out["top_logp"], val, np.take_along_axis(off, np.maximum(idx, 0), 1))


def backward(x, targets, rmax, rlog, dlogp, scale=1.0, entropy=None, dentropy=None, dx=None):
    return grass.logp_backward(x, targets, rmax, rlog, dlogp, nan(x.shape, x.dtype) if dx is None else dx, scale, entropy=entropy,
                               dentropy=dentropy)


def check_backward(x, targets, rmax, rlog, dlogp, scale, entropy, dentropy, dx, steps=4, least=TINY):
    T = x.shape[0]
    f = lambda v: np.zeros(T) if v is None else to_f64(v)  # noqa: E731
    ids = np.full(T, -1) if targets is None or dlogp is None else targets.cpu().numpy().astype(np.int64)
    m, r, g, H, h = f(rmax), f(rlog), f(dlogp), f(entropy), f(dentropy)
    want, l, p = ends_ref.logp_backward(to_f64(x), ids, scale, m, r, g, H, h)
    with np.errstate(all="ignore"):
        arg = np.abs(l + r[:, None]) + np.abs(r)[:, None]
        rel = (steps * arg + 8) * U
        lH = np.abs(l) + np.abs(H)[:, None]
        size = np.abs(g)[:, None] * (p * rel + 2 * U * p) + np.abs(h)[:, None] * p * (lH * (rel + 4 * U) + 4 * U * (arg + lH))
        size = np.where(p == 0, 0.0, size)
        there = (ids >= 0) & (ids < x.shape[1])
        size[there, ids[there]] += 4 * U * np.abs(g[there])
        size = size * scale + 2 * U * np.abs(want)
        half = torch.finfo(x.dtype).eps / 2 if x.dtype == BF16 else 0.0
        off = size + half * (np.abs(want) + size) + least * (1 + np.abs(g) + np.abs(h))[:, None]
    assert near(dx, want, off)


VOCABULARIES = [1, 2, 3, 5, 7, 8, 9, 31, 63, 64, 65, 100, 255, 256, 257, 511, 512, 513, 520, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4097,
                8191, 8192, 8200, 16383, 16385, 32000, 32769, 50001, 65535, 65536, 65537, 70001, 131071, 131073, 140000, 262144, 300001]
CASES = [(V, (1, 2, 5, 3)[(i + j) % 4], dt, (0, 1, 5, 20, 33, 64)[(i + 2 * j) % 6]) for i, V in enumerate(VOCABULARIES)
         for j, dt in enumerate((F32, BF16))]


@pytest.mark.parametrize("V,T,dtype,top", CASES)
def test_forward_and_backward(V, T, dtype, top):
    x = draw((T, V), 1, dtype, 3.0)
    targets = whole((T,), 2, V).to((torch.int32, torch.int64)[V % 2])
    scale = (1.0, float(np.float32(0.7)))[V % 3 == 0]
    out = forward(x, targets, min(top, V), scale)
    check_forward(x, targets, scale, out)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    for entropy, d in ((None, None), (out["entropy"], dH)):
        dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, scale, entropy, d)
        check_backward(x, targets, out["rmax"], out["rlog"], dlogp, scale, entropy, d, dx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,more,offset", [(1, 1, 1), (5, 1, 1), (100, 3, 1), (512, 8, 8), (513, 2, 3), (3001, 1, 1), (20000, 5, 7), (50001, 7, 7),
                                           (140001, 3, 5)])
def test_rows_in_any_position(V, more, offset, dtype):
    """Rows inside larger arrays, on any boundary: nothing around them is read for a result (it holds plus infinity), or written."""
    T = 6
    x, targets = draw((T, V), 1, dtype, 2.0), whole((T,), 2, V)
    vx, _ = padded(x, V + more, offset)
    out = forward(vx, targets, min(V, 9))
    check_forward(x, targets, 1.0, out)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    vd, fd = padded(nan((T, V), dtype), V + more + 1, offset + 2)
    backward(vx, targets, out["rmax"], out["rlog"], dlogp, 1.0, out["entropy"], dH, vd)
    check_backward(x, targets, out["rmax"], out["rlog"], dlogp, 1.0, out["entropy"], dH, vd.contiguous())
    assert int((fd == INF).sum()) == fd.numel() - vd.numel()
    backward(vx, targets, out["rmax"], out["rlog"], dlogp, 1.0, out["entropy"], dH, vx)
    assert torch.equal(vx, vd), "in place"


def special(V, dtype, seed):
    """Rows where it can go wrong, and what they are."""
    low = torch.finfo(dtype).min
    base = draw((V,), seed, dtype, 3.0)
    j = torch.arange(V, device=DEV)
    few = torch.full((V,), -INF, dtype=dtype, device=DEV)
    few[j % max(1, V // 3) == V // 7] = 1.5
    lowest = torch.full((V,), low, dtype=dtype, device=DEV)
    lowest[[V // 2, V - 1]] = base[:2]
    rows = {"plain": base, "all masked": torch.full_like(base, -INF), "one left": torch.where(j == V - 1, base, -INF), "few left": few,
            "all at the lowest": torch.full_like(base, low), "few above the lowest": lowest, "constant": torch.full_like(base, 0.25),
            "two values": (j % 2).to(dtype), "ties at the end": torch.where(j >= V - 3 * V // 4, 2.0, base.float().clamp(max=1.0)).to(dtype),
            "rising": (j / V * 8).to(dtype), "falling": (-j / V * 8).to(dtype), "zeros of both signs": torch.where(j % 3 == 0, -0.0, 0.0).to(dtype),
            "peaks far apart": torch.where(j % 512 < 8, 6.0 + (j % 97) / 97, base.float()).to(dtype),
            "peaks farther apart": torch.where(j % 8192 < 8, 6.0 + (j % 89) / 97, base.float()).to(dtype),
            "large": (base.float() * 1e4).to(dtype), "huge": torch.where(j % 5 == 0, -low, base.float() * 1e37).to(dtype),
            "a NaN": torch.where(j == V // 3, NAN, base), "all NaN": torch.full_like(base, NAN), "an infinity": torch.where(j == V // 2, INF, base),
            "infinities of both signs": torch.where(j == V // 2, INF, torch.where(j % 2 == 0, -INF, base)),
            "a NaN among masked": torch.where(j == 0, NAN, -INF).to(dtype), "masked but for its first": torch.where(j == 0, base, -INF)}
    return list(rows), torch.stack([r.to(dtype) for r in rows.values()])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [4, 37, 300, 512, 1500, 4096, 9000, 32000, 70000, 140003])
@pytest.mark.parametrize("top", [1, 16, 20, 64])
def test_special_rows(V, dtype, top):
    top = min(top, V)
    names, x = special(V, dtype, V)
    T = len(names)
    targets = whole((T,), 5, V)
    targets[3], targets[7] = -100, V
    out = forward(x, targets, top, 0.5)
    check_forward(x, targets, 0.5, out)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    for entropy, d in ((None, None), (out["entropy"], dH)):
        dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, 0.5, entropy, d)
        check_backward(x, targets, out["rmax"], out["rlog"], dlogp, 0.5, entropy, d, dx)
    assert not dx[names.index("all masked")].any()


@pytest.mark.parametrize("V", [90, 2000, 33000, 150001])
def test_rows_without_a_gradient_are_zeros_and_are_not_read(V):
    T = 9
    x, targets = draw((T, V), 1, BF16, 2.0), whole((T,), 2, V)
    out = forward(x, targets, 0)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    targets[1], dlogp[2], targets[4] = -100, 0.0, V
    dH[1] = dH[2] = 0.0
    x[1], x[2] = NAN, INF
    dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, 1.0, out["entropy"], dH)
    assert not dx[1:3].any() and bool(dx[4].any())
    keep = [0, 3, 4, 5, 6, 7, 8]
    check_backward(x[keep], targets[keep], out["rmax"][keep], out["rlog"][keep], dlogp[keep], 1.0, out["entropy"][keep], dH[keep], dx[keep])
    assert not backward(x, None, out["rmax"], out["rlog"], None).any()
    dx = backward(x[keep], None, out["rmax"][keep], out["rlog"][keep], None, 1.0, out["entropy"][keep], dH[keep])
    check_backward(x[keep], None, out["rmax"][keep], out["rlog"][keep], None, 1.0, out["entropy"][keep], dH[keep], dx)


@pytest.mark.parametrize("V", [50, 1000, 40000, 200000])
def test_outputs_by_themselves(V):
    x, targets = draw((3, V), 1, BF16, 2.0), whole((3,), 2, V)
    all_of_it = forward(x, targets, 7)
    check_forward(x, targets, 1.0, all_of_it)
    for kw in (dict(top=0, entropy=False, keep=False), dict(top=7, entropy=False, keep=False), dict(top=0, entropy=True, keep=False),
               dict(top=0, entropy=False, keep=True)):
        for t in (targets, None):
            out = forward(x, t, kw["top"], entropy=kw["entropy"], keep=kw["keep"])
            for name, got in out.items():
                assert got is None or torch.equal(got, all_of_it[name]), (name, kw)


@pytest.mark.parametrize("T,V,dtype", [(1500, 50, F32), (3000, 300, BF16), (700, 3000, F32), (1300, 9000, BF16), (600, 33000, BF16),
                                       (600, 70001, F32), (300, 140000, BF16)])
def test_more_rows_than_workgroups(T, V, dtype):
    """Against torch in 64 bits on the card, since such arrays are large; the bounds are the largest over the rows."""
    x, targets = draw((T, V), 1, dtype, 2.0), whole((T,), 2, V)
    out = forward(x, targets, 3)
    logp = torch.log_softmax(x.double(), 1)
    H = torch.special.entr(logp.exp()).sum(1)
    big = float(264 + 4 * np.log(V) * 2 + 4 * float(logp.abs().max())) * U
    assert float((out["logp"].double() - logp.gather(1, targets.view(-1, 1))[:, 0]).abs().max()) <= big
    assert float((out["entropy"].double() - H).abs().max()) <= big * (1 + np.log(V))
    assert torch.equal(out["rmax"], x.float().amax(1))
    order = (x.float() + 0.0).view(torch.int32)
    order = torch.where(order < 0, order ^ 0x7FFFFFFF, order).long() * (1 << 32) - torch.arange(V, device=DEV)
    assert torch.equal(out["top_idx"].long(), torch.topk(order, 3, dim=1).indices)
    dlogp = draw((T,), 3, F32)
    dx = backward(x, targets, out["rmax"], out["rlog"], dlogp).double()
    want = -dlogp.double().view(-1, 1) * logp.exp()
    want.scatter_add_(1, targets.view(-1, 1), dlogp.double().view(-1, 1))
    half = torch.finfo(dtype).eps / 2
    off = (2 * half + big * 2) * want.abs() + 2 * big * dlogp.abs().double().view(-1, 1) * logp.exp() + 4 * U * dlogp.abs().max()
    assert bool(((dx - want).abs() <= off).all())
    again = forward(x, targets, 3)
    assert all(torch.equal(out[k], again[k]) for k in out), "equal calls give equal bits"


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_very_long_row(dtype):
    V = 5000011
    x, targets = draw((2, V), 1, dtype, 2.0), torch.tensor([V - 1, 3], device=DEV)
    out = forward(x, targets, 64)
    check_forward(x, targets, 1.0, out)


def test_offsets_beyond_32_bits():
    ld, V = (1 << 30) + 8, 40000
    room = torch.empty(3 * ld + V, dtype=BF16, device=DEV)
    x, targets = draw((4, V), 1, BF16, 2.0), whole((4,), 2, V)
    view = torch.as_strided(room, (4, V), (ld, 1))
    view.copy_(x)
    out = forward(view, targets, 5)
    check_forward(x, targets, 1.0, out)
    dlogp = draw((4,), 3, F32)
    want = backward(x, targets, out["rmax"], out["rlog"], dlogp)
    assert torch.equal(backward(view, targets, out["rmax"], out["rlog"], dlogp, dx=view), want)


def test_target_numbers_of_64_bits_are_not_cut():
    x = draw((5, 100), 1, F32)
    targets = torch.tensor([3, (1 << 32) + 3, -(1 << 32) + 3, 1 << 62, -(1 << 63)], device=DEV)
    out = forward(x, targets, 0)
    check_forward(x, targets, 1.0, out)
    assert float(out["logp"][0]) != 0 and not out["logp"][1:].any()
    assert not backward(x, targets, out["rmax"], out["rlog"], torch.ones(5, device=DEV))[1:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 5000, 70001])
@pytest.mark.parametrize("scale", [3e38, 1e30, 1e6, 1e-6, 1e-30, 1e-38])
def test_temperatures_of_any_size(V, scale, dtype):
    """Cold ones leave the largest logits alone (here with a tie), hot ones make all alike."""
    x = draw((4, V), 1, dtype, 2.0)
    x[1, V // 2] = x[1].max()
    x[2] = x[2] * 1e30
    x[3, 1:] = -INF
    targets = torch.stack([x[0].argmax(), x[1].argmax(), x[2].argmin(), torch.zeros((), dtype=torch.int64, device=DEV)])
    scale = float(np.float32(scale))
    out = forward(x, targets, min(V, 4), scale)
    check_forward(x, None, scale, {**out, "top_logp": None, "top_idx": None})
    _, rlog, logp, H = ends_ref.logp_rows(to_f64(x), scale)
    idx, val = ends_ref.alternatives(to_f64(x), logp, min(V, 4))
    assert np.array_equal(out["top_idx"].cpu().numpy(), idx)
    for got, want in ((out["logp"], ends_ref.given(logp, targets.cpu().numpy())), (out["top_logp"], val)):
        beyond = (want < -3.3e38) & (to_f64(got) < -3.3e38)  # where fp32 ends
        size = (264 + 3 * (H - rlog) + 9 * rlog).reshape(4, *[1] * (want.ndim - 1))
        with np.errstate(all="ignore"):
            assert near(torch.from_numpy(np.where(beyond, 0.0, to_f64(got))), np.where(beyond, 0.0, want), (size + 4 * np.abs(want)) * U)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 5000, 70001])
@pytest.mark.parametrize("scale", [3e38, 1e30, 1e6, 1e-6, 1e-30, 1e-38])
def test_gradient_at_temperatures_of_any_size(V, scale, dtype):
    """The difference of two logits, scale log2(e), their product and the difference with rlog are rounded: five halves of a step.
    Probabilities below 2^-126 may be zero, times the scale, and times their logarithm below 128."""
    x = draw((4, V), 1, dtype, 2.0)
    x[1, V // 2] = x[1].max()
    x[2] = x[2] * 1e30
    x[3, 1:] = -INF
    targets = torch.stack([x[0].argmax(), x[1].argmax(), x[2].argmin(), torch.zeros((), dtype=torch.int64, device=DEV)])
    scale = float(np.float32(scale))
    out = forward(x, targets, 0, scale)
    dlogp, dH = draw((4,), 3, F32).clamp(-1, 1), draw((4,), 4, F32).clamp(-1, 1) / 300
    dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, scale, out["entropy"], dH)
    check_backward(x, targets, out["rmax"], out["rlog"], dlogp, scale, out["entropy"], dH, dx, 5, 2 * TINY * max(1.0, scale))


def test_gradient_against_differences():
    """Along random directions v, |v| <= 1, in fp32 through the kernels, over a step of 1/16 to both sides: (1/16)^2 / 6 of the
    third derivative is left.  For log p that is the third central moment of v, below 1; for the entropy the joint cumulant of x and
    three times v, at most std(x) (4 std(v) + 3 std(v)^3), and three third moments: below 8 at std(x) near 1 and std(v) below a
    half.  The difference of two values of size below 8 is off by 2 * 300 U * 8, over 1/8."""
    T, V = 6, 700
    x, targets = draw((T, V), 1, F32), whole((T,), 2, V)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    out = forward(x, targets, 0)
    dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, 1.0, out["entropy"], dH)
    for seed in range(5):
        v = draw((T, V), 10 + seed, F32)
        v /= v.abs().amax(1, keepdim=True)
        a, b = (forward(x + s * v / 16, targets, 0) for s in (1, -1))
        slope = (dlogp * (a["logp"] - b["logp"]) + dH * (a["entropy"] - b["entropy"])).double() * 8
        off = (dlogp.abs() + 8 * dH.abs()).double() * (1 / 256 / 6 + 2 * 300 * U * 8 * 8)
        assert bool(((dx.double() * v).sum(1) - slope).abs().le(off).all())


@pytest.mark.parametrize("T,V", [(5, 900), (3, 40000), (2, 200000)])
def test_on_another_stream_and_in_a_graph(T, V):
    a, b = draw((T, V), 1, BF16, 2.0), draw((T, V), 2, BF16, 3.0)
    ta, tb = whole((T,), 3, V), whole((T,), 4, V)
    dlogp, dH = draw((T,), 5, F32), draw((T,), 6, F32)
    x, targets, dx = a.clone(), ta.clone(), nan((T, V), BF16)
    logp, entropy, rmax, rlog, tl = nan((T,)), nan((T,)), nan((T,)), nan((T,)), nan((T, 6))
    ti = torch.zeros((T, 6), dtype=torch.int32, device=DEV)
    ws = grass.workspace(grass.logp_forward_workspace(T, V, 6, grass.BF16))

    def both():
        grass.logp_forward(x, targets, logp, ws, 1.5, entropy=entropy, rmax=rmax, rlog=rlog, top_logp=tl, top_idx=ti)
        grass.logp_backward(x, targets, rmax, rlog, dlogp, dx, 1.5, entropy=entropy, dentropy=dH)

    def check(z, t):
        check_forward(z, t, 1.5, dict(logp=logp, entropy=entropy, rmax=rmax, rlog=rlog, top_logp=tl, top_idx=ti))
        check_backward(z, t, rmax, rlog, dlogp, 1.5, entropy, dH, dx)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    check(a, ta)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(4):
        z, t = ((b, tb), (a, ta))[turn % 2]
        x.copy_(z)
        targets.copy_(t)
        for out in (logp, entropy, rmax, rlog, tl, dx):
            out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        check(z, t)
        eager = forward(z, t, 6, 1.5)
        assert torch.equal(eager["logp"], logp) and torch.equal(eager["top_idx"], ti)


def test_binding_refuses():
    x, t, f = draw((4, 12), 1, F32), whole((4,), 2, 12), nan((4,))
    ws, i = grass.workspace(1 << 16), torch.zeros((4, 3), dtype=torch.int32, device=DEV)
    for bad in (lambda: grass.logp_forward(x.t(), t, f, ws), lambda: grass.logp_forward(x, t.float(), f, ws), lambda: grass.logp_forward(x, t, f[:3], ws),
                lambda: grass.logp_forward(x, t, f, ws, top_logp=nan((4, 2)), top_idx=i), lambda: grass.logp_forward(x, t, f, ws, entropy=f.double()),
                lambda: grass.logp_forward(x, t, f, ws, top_logp=nan((4, 3)), top_idx=i.long()), lambda: grass.logp_forward(x.half(), t, f, ws),
                lambda: grass.logp_forward(nan((1, 24))[:, ::2], t[:1], f[:1], ws), lambda: grass.logp_forward(x, t.cpu(), f, ws),
                lambda: grass.logp_backward(x, t, f, f, f, nan((4, 11))), lambda: grass.logp_backward(x, t, f, f, f, nan((4, 12), BF16)),
                lambda: grass.logp_backward(x, t[:2], f, f, f, nan((4, 12)))):
        with pytest.raises((AssertionError, TypeError)):
            bad()
    for bad in (lambda: grass.logp_forward(x, t, None, ws), lambda: grass.logp_forward(x, t, f, ws, 0.0),
                lambda: grass.logp_backward(x, t, None, f, f, nan((4, 12)))):
        with pytest.raises(grass.GrassError):
            bad()
