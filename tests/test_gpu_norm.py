"""grass_norm_forward and grass_norm_backward against the same formulas in 64 bits.

Tolerances.  An output is rounded once to its type: half a step, finfo.eps / 2 of its value.  What
comes before is fp32: a row's sum runs through at most 64 values in a lane (80 in the loops over
wide rows used here) and then a tree, so that its error is below 100 half steps of fp32 of the sum of
the magnitudes; the other operations add a few.  FP32 = 128 * 2^-24 of the magnitudes that
enter an output covers both.  Sums over tokens run through at most T terms, or 300 + T / 256 where
many rows are summed by several workgroups."""
import os
import re

import numpy as np
import pytest
import torch

import norm_ref
from gpu_util import DEV, to_f64
from paper_2406_17660_amd import grass

pytestmark = pytest.mark.gpu
EPS = 1e-5
FP32 = 128 * 2.0 ** -24
KINDS = {"layer": grass.NORM_LAYER, "rms": grass.NORM_RMS}
WIDTHS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 127, 128, 129, 383, 511, 512, 513, 520, 1000, 1024, 1025, 1293, 2047, 2048, 2049,
          2056, 4095, 4096, 4097, 5461, 8191, 8192, 8200, 12289, 16383, 16384, 16385, 20000]


def draw(shape, seed, dtype, scale=1.0, shift=0.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale + shift).to(dtype)


def padded(t, ld, offset):
    """The values of t in rows ld elements apart, the first `offset` elements behind the base; everything
    around them is NaN."""
    T, n = t.shape
    flat = torch.full((offset + T * ld + 8,), float("nan"), dtype=t.dtype, device=DEV)
    view = flat[offset:offset + T * ld].view(T, ld)[:, :n]
    view.copy_(t)
    return view, flat


def half(dtype):
    return torch.finfo(dtype).eps / 2


def check_forward(X, R, gain, bias, kind, Y, H, mean, rstd, eps=EPS):
    dt = X.dtype
    h = to_f64(X)
    if R is not None:
        want_h = (X.float() + R.float()).to(dt)
        assert torch.equal(H, want_h)
        h = to_f64(want_h)
    g, b = (None if v is None else to_f64(v) for v in (gain, bias))
    y, mu, rs = norm_ref.forward(h, g, b, eps, kind == "layer")
    size = np.abs(h).mean(1)[:, None] * rs[:, None] * (1.0 if g is None else np.abs(g)) + np.abs(y)
    if b is not None:
        size = size + np.abs(b)
    assert (np.abs(to_f64(Y) - y) <= half(dt) * np.abs(y) * (1 + FP32) + FP32 * size).all()
    if mean is not None:
        assert (np.abs(to_f64(mean) - mu) <= FP32 * np.abs(h).mean(1)).all()
    if rstd is not None:
        # (the mean's error moves the squares about it by its square alone)
        off = (FP32 * np.abs(h).mean(1) * rs) ** 2
        assert (np.abs(to_f64(rstd) - rs) <= (FP32 + off) * rs).all()


def depth(T):
    return min(T, 300 + T / 256) + 16


def check_backward(dY, H, gain, mean, rstd, kind, dR, dX, dgain, dbias):
    dt = dY.dtype
    dy, h, rs = to_f64(dY), to_f64(H), to_f64(rstd)
    mu = to_f64(mean) if mean is not None else np.zeros(len(rs))
    g = None if gain is None else to_f64(gain)
    dx, dg, db = norm_ref.backward(dy, h, g, mu, rs, kind == "layer")
    xh = (h - mu[:, None]) * rs[:, None]
    z = dy if g is None else dy * g
    size = rs[:, None] * (np.abs(z) + np.abs(z).mean(1)[:, None] + np.abs(xh) * np.abs(z * xh).mean(1)[:, None])
    if dR is not None:
        dx = dx + to_f64(dR)
        size = size + np.abs(to_f64(dR))
    assert (np.abs(to_f64(dX) - dx) <= half(dt) * np.abs(dx) * (1 + FP32) + FP32 * size).all()
    if dgain is not None:
        assert (np.abs(to_f64(dgain) - dg) <= depth(len(rs)) * 2.0 ** -24 * np.abs(dy * xh).sum(0)).all()
    if dbias is not None:
        assert (np.abs(to_f64(dbias) - db) <= depth(len(rs)) * 2.0 ** -24 * np.abs(dy).sum(0)).all()


def stats(H, kind, eps=EPS):
    _, mu, rs = norm_ref.forward(to_f64(H), None, None, eps, kind == "layer")
    f = lambda a: torch.tensor(a, dtype=torch.float32, device=DEV)  # noqa: E731
    return (f(mu) if kind == "layer" else None), f(rs)


def nan(shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def code(dtype):
    return grass.F32 if dtype == torch.float32 else grass.BF16


def gpu_backward(dY, H, gain, mean, rstd, kind, dR=None, dX=None, want=("dgain", "dbias")):
    T, n = dY.shape
    dX = nan((T, n), dY.dtype) if dX is None else dX
    dgain = nan((n,)) if "dgain" in want else None
    dbias = nan((n,)) if "dbias" in want else None
    ws = grass.workspace(grass.norm_backward_workspace(T, n, code(dY.dtype)))
    ws.view(torch.uint8).fill_(0xFF)
    grass.norm_backward(dY, H, gain, mean, rstd, dX, dgain, dbias, ws, KINDS[kind], dR=dR)
    return dX, dgain, dbias


CASES = []
for _i, _n in enumerate(WIDTHS):
    for _j, (_dt, _kind) in enumerate([(d, k) for d in (torch.float32, torch.bfloat16) for k in ("layer", "rms")]):
        CASES.append((_n, (1, 2, 5, 19, 70)[(_i + _j) % 5], _dt, _kind, (_i + _j) % 4, _i % 2 == 0))


@pytest.mark.parametrize("n,T,dtype,kind,vectors,add", CASES)
def test_forward(n, T, dtype, kind, vectors, add):
    gdt = torch.float32 if vectors % 2 else torch.bfloat16
    gain = draw(n, 1, gdt, 0.2, 1.0) if vectors else None
    bias = draw(n, 2, gdt, 0.2) if vectors >= 2 else None
    X = draw((T, n), 3, dtype, 1.5, 0.4)
    R = draw((T, n), 4, dtype) if add else None
    Y, H = nan((T, n), dtype), nan((T, n), dtype) if add else None
    mean, rstd = nan((T,)), nan((T,))
    grass.norm_forward(X, gain, bias, EPS, Y, KINDS[kind], R=R, H=H, mean=mean, rstd=rstd)
    check_forward(X, R, gain, bias, kind, Y, H, mean if kind == "layer" else None, rstd)


@pytest.mark.parametrize("n,T,dtype,kind,vectors,add", CASES)
def test_backward(n, T, dtype, kind, vectors, add):
    gdt = torch.float32 if vectors % 2 else torch.bfloat16
    gain = draw(n, 1, gdt, 0.2, 1.0) if vectors else None
    dY, H = draw((T, n), 5, dtype, 0.3, 0.05), draw((T, n), 6, dtype, 1.5, 0.4)
    dR = draw((T, n), 7, dtype, 0.3) if add else None
    mean, rstd = stats(H, kind)
    want = (("dgain", "dbias"), ("dgain",), ("dbias",), ("dgain", "dbias"))[vectors]
    dX, dgain, dbias = gpu_backward(dY, H, gain, mean, rstd, kind, dR, want=want)
    check_backward(dY, H, gain, mean, rstd, kind, dR, dX, dgain, dbias)


@pytest.mark.parametrize("T,n,dtype", [(1024, 64, torch.bfloat16), (4099, 128, torch.float32), (4100, 512, torch.bfloat16),
                                       (3001, 1000, torch.bfloat16), (2600, 2056, torch.float32),
                                       (1500, 4096, torch.bfloat16), (1100, 5461, torch.bfloat16), (1030, 16385, torch.bfloat16)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_more_rows_than_workgroups(T, n, dtype, kind):
    gain, bias = draw(n, 1, torch.float32, 0.2, 1.0), draw(n, 2, torch.float32, 0.2)
    X = draw((T, n), 3, dtype, 1.5, 0.4)
    Y, mean, rstd = nan((T, n), dtype), nan((T,)), nan((T,))
    grass.norm_forward(X, gain, bias, EPS, Y, KINDS[kind], mean=mean, rstd=rstd)
    check_forward(X, None, gain, bias, kind, Y, None, mean if kind == "layer" else None, rstd)
    dY = draw((T, n), 5, dtype, 0.3, 0.05)
    first = gpu_backward(dY, X, gain, mean, rstd, kind)
    check_backward(dY, X, gain, mean if kind == "layer" else None, rstd, kind, None, *first)
    for again, was in zip(gpu_backward(dY, X, gain, mean, rstd, kind), first):
        assert torch.equal(again, was), "equal calls give equal bits"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,more,offset", [(5, 1, 1), (100, 3, 1), (512, 8, 8), (513, 2, 3), (1293, 1, 1), (4096, 5, 7), (9000, 3, 1),
                                           (17001, 1, 1)])
def test_rows_in_any_position(n, more, offset, dtype):
    """Rows inside larger arrays, on any boundary; nothing around them is read or written."""
    T, kind = 6, "layer"
    gain, bias = draw(n + 1, 1, dtype, 0.2, 1.0)[1:], draw(n + 1, 2, dtype, 0.2)[1:]
    X, R = draw((T, n), 3, dtype, 1.5, 0.4), draw((T, n), 4, dtype)
    vX, _ = padded(X, n + more, offset)
    vR, _ = padded(R, n + more + 2, offset + 1)
    (vH, fH), (vY, fY) = padded(nan((T, n), dtype), n + more + 1, offset + 2), padded(nan((T, n), dtype), n + more, offset)
    mean, rstd = nan((T,)), nan((T,))
    grass.norm_forward(vX, gain, bias, EPS, vY, KINDS[kind], R=vR, H=vH, mean=mean, rstd=rstd)
    check_forward(X, R, gain, bias, kind, vY.contiguous(), vH.contiguous(), mean, rstd)
    for flat, view in ((fH, vH), (fY, vY)):
        assert int((~torch.isnan(flat.float())).sum()) == view.numel()
    dY, dR = draw((T, n), 5, dtype, 0.3), draw((T, n), 7, dtype, 0.3)
    vdY, _ = padded(dY, n + more, offset)
    vdR, _ = padded(dR, n + more + 1, offset + 2)
    vdX, fdX = padded(nan((T, n), dtype), n + more + 3, offset + 1)
    _, dgain, dbias = gpu_backward(vdY, vH, gain, mean, rstd, kind, vdR, vdX)
    check_backward(dY, vH.contiguous(), gain, mean, rstd, kind, dR, vdX.contiguous(), dgain, dbias)
    assert int((~torch.isnan(fdX.float())).sum()) == vdX.numel()


@pytest.mark.parametrize("n", [40, 600, 4096, 20000])
def test_outputs_in_place(n):
    T, dt = 9, torch.bfloat16
    gain, bias = draw(n, 1, dt, 0.2, 1.0), draw(n, 2, dt, 0.2)
    X, R = draw((T, n), 3, dt, 1.5, 0.4), draw((T, n), 4, dt)
    want_H, want_Y = torch.empty_like(X), torch.empty_like(X)
    mean, rstd = nan((T,)), nan((T,))
    grass.norm_forward(X, gain, bias, EPS, want_Y, R=R, H=want_H, mean=mean, rstd=rstd)
    for h, y in (("X", "R"), ("R", "X"), ("X", None), (None, "X"), (None, "R")):
        a = {"X": X.clone(), "R": R.clone(), None: torch.empty_like(X)}
        Y = a[y] if y else torch.empty_like(X)
        H = a[h] if h else torch.empty_like(X)
        grass.norm_forward(a["X"], gain, bias, EPS, Y, R=a["R"], H=H)
        assert torch.equal(Y, want_Y) and torch.equal(H, want_H)
    alone = X.clone()
    grass.norm_forward(alone, gain, bias, EPS, alone)
    want = torch.empty_like(X)
    grass.norm_forward(X, gain, bias, EPS, want)
    assert torch.equal(alone, want)
    dY, dR = draw((T, n), 5, dt, 0.3), draw((T, n), 7, dt, 0.3)
    want = gpu_backward(dY, want_H, gain, mean, rstd, "layer", dR)
    for which in range(3):
        a = [dY.clone(), want_H.clone(), dR.clone()]
        got = gpu_backward(a[0], a[1], gain, mean, rstd, "layer", a[2], dX=a[which])
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("T,n,dtype", [(2000, 1293, torch.float32), (1500, 2055, torch.bfloat16), (900, 4097, torch.bfloat16),
                                       (1200, 8193, torch.bfloat16), (500, 9001, torch.float32)])
def test_outputs_in_place_where_rows_start_anywhere(T, n, dtype):
    """Rows that several wavefronts share and whose last vector lies over the one before: dX over each of its
    inputs, and H and Y over theirs, give what separate arrays give."""
    gain = draw(n, 1, torch.float32, 0.2, 1.0)
    X, R, dY, dR = (draw((T, n), k, dtype) for k in (3, 4, 5, 7))
    H, Y, mean, rstd = torch.empty_like(X), torch.empty_like(X), nan((T,)), nan((T,))
    grass.norm_forward(X, gain, None, EPS, Y, R=R, H=H, mean=mean, rstd=rstd)
    a, b = X.clone(), R.clone()
    grass.norm_forward(a, gain, None, EPS, a, R=b, H=b)
    assert torch.equal(a, Y) and torch.equal(b, H)
    want = gpu_backward(dY, H, gain, mean, rstd, "layer", dR)
    for which in range(3):
        a = [dY.clone(), H.clone(), dR.clone()]
        got = gpu_backward(a[0], a[1], gain, mean, rstd, "layer", a[2], dX=a[which])
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("n", [9, 1024, 4097, 17000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_that_are_not_finite_stay_in_their_row(n, dtype):
    T = 6
    X = draw((T, n), 3, dtype, 1.5, 0.4)
    clean = X.clone()
    X[1, n // 2], X[3, 0], X[4, n - 1] = float("nan"), float("inf"), float("-inf")
    Y, want = nan((T, n), dtype), nan((T, n), dtype)
    for kind in KINDS:
        grass.norm_forward(X, None, None, EPS, Y, KINDS[kind])
        grass.norm_forward(clean, None, None, EPS, want, KINDS[kind])
        for t in (0, 2, 5):
            assert torch.equal(Y[t], want[t])
        assert torch.isnan(Y[1]).all() and torch.isnan(Y[3]).any() and torch.isnan(Y[4]).any()
        if kind == "layer":
            assert torch.isnan(Y[3]).all() and torch.isnan(Y[4]).all()


def test_rows_without_spread_and_far_means():
    """A constant row is the bias (its variance is zero); a row whose mean is a thousand times its spread
    keeps the spread's digits."""
    n = 1000
    X = torch.full((2, n), 3.25, device=DEV)
    X[1] = draw(n, 8, torch.float32, 1.0, 1000.0)
    bias = draw(n, 2, torch.float32)
    Y, mean, rstd = nan((2, n)), nan((2,)), nan((2,))
    grass.norm_forward(X, None, bias, EPS, Y, mean=mean, rstd=rstd)
    assert torch.equal(Y[0], bias) and abs(rstd[0].item() - EPS ** -0.5) < 1e-4 * EPS ** -0.5
    check_forward(X, None, None, bias, "layer", Y, None, mean, rstd)


def test_no_rows():
    n = 100
    e = torch.empty((0, n), device=DEV)
    grass.norm_forward(e, None, None, EPS, e.clone())
    _, dgain, dbias = gpu_backward(e, e, None, torch.empty(0, device=DEV), torch.empty(0, device=DEV), "layer")
    assert (dgain == 0).all() and (dbias == 0).all()


def test_forward_against_differences_of_the_kernel_itself():
    """The kernel's gradients against central differences of the kernel's own forward pass (fp32: steps of
    2^-6, whose curvature and rounding stay below 2e-3 of a loss of a few units)."""
    T, n, step = 3, 33, 2.0 ** -6
    X, gain, bias, dY = draw((T, n), 3, torch.float32), draw(n, 1, torch.float32, 0.2, 1.0), draw(n, 2, torch.float32), \
        draw((T, n), 5, torch.float32)
    for kind in KINDS:
        Y, mean, rstd = torch.empty_like(X), nan((T,)), nan((T,))

        def loss():
            grass.norm_forward(X, gain, bias, EPS, Y, KINDS[kind], mean=mean, rstd=rstd)
            return float((Y.double() * dY.double()).sum())

        loss()
        got = gpu_backward(dY, X, gain, mean, rstd, kind)
        for of, grad in zip((X, gain, bias), got):
            flat, g = of.view(-1), grad.view(-1).cpu()
            for k in range(0, flat.numel(), 7):
                was = flat[k].item()
                flat[k] = was + step
                up = loss()
                flat[k] = was - step
                down = loss()
                flat[k] = was
                assert abs((up - down) / (2 * step) - g[k].item()) < 2e-3 * (1 + abs(g[k].item()))


def test_side_stream_and_graph():
    """On a stream of its own, and captured: every replay equals the eager result, with eager work between."""
    T, n, dt = 300, 1024, torch.bfloat16
    gain = draw(n, 1, torch.float32, 0.2, 1.0)
    X, R, dY, dR = (draw((T, n), k, dt) for k in (3, 4, 5, 7))
    out = {k: nan((T, n), dt) for k in ("H", "Y", "dX")}
    rstd, dgain = nan((T,)), nan((n,))
    ws = grass.workspace(grass.norm_backward_workspace(T, n, grass.BF16))

    def both():
        grass.norm_forward(X, gain, None, EPS, out["Y"], grass.NORM_RMS, R=R, H=out["H"], rstd=rstd)
        grass.norm_backward(dY, out["H"], gain, None, rstd, out["dX"], dgain, None, ws, grass.NORM_RMS, dR=dR)

    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (*out.values(), rstd, dgain)]
    side = torch.cuda.Stream()
    for t in (*out.values(), rstd, dgain):
        t.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((*out.values(), rstd, dgain), want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (*out.values(), rstd, dgain):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out.values(), rstd, dgain), want))


def test_rows_beyond_32_bit_offsets():
    """Rows 2^30 + 8 elements apart: the third starts behind 2^31 elements, 2^32 bytes."""
    T, n, ld, dt = 3, 4096, (1 << 30) + 8, torch.bfloat16
    far = lambda: torch.zeros(2 * ld + n, dtype=dt, device=DEV).as_strided((T, n), (ld, 1))  # noqa: E731
    X, dY = far(), far()
    X.copy_(draw((T, n), 3, dt, 1.5, 0.4))
    dY.copy_(draw((T, n), 5, dt, 0.3))
    mean, rstd = nan((T,)), nan((T,))
    Y = far()
    grass.norm_forward(X, None, None, EPS, Y, mean=mean, rstd=rstd)
    check_forward(X.contiguous(), None, None, None, "layer", Y.contiguous(), None, mean, rstd)
    dX, dgain, dbias = gpu_backward(dY, X, None, mean, rstd, "layer", dX=Y)
    check_backward(dY.contiguous(), X.contiguous(), None, mean, rstd, "layer", None, dX.contiguous(), dgain, dbias)


@pytest.mark.parametrize("T", [0, 1])
def test_more_columns_than_a_grid_of_their_sums_has_threads_for(T):
    """16 threads for each column's sum: 2^28 columns are 2^32 threads.  One row: its sums are single products."""
    n = (1 << 28) + 100
    gen = torch.Generator(device=DEV)
    gen.manual_seed(11)
    dY, H = (torch.empty((T, n), dtype=torch.bfloat16, device=DEV).normal_(generator=gen) for _ in range(2))
    rstd = torch.full((T,), 0.5, device=DEV)
    dX, dgain, dbias = gpu_backward(dY, H, None, None, rstd, "rms")
    if T == 0:
        assert int(torch.count_nonzero(dgain)) == 0 and int(torch.count_nonzero(dbias)) == 0
        return
    assert torch.equal(dbias, dY[0].float())
    assert torch.equal(dgain, dY[0].float() * (H[0].float() * 0.5))
    assert torch.isfinite(dX).all()


@pytest.mark.parametrize("T,n,dtype", [(769, 64, torch.bfloat16), (1999, 250, torch.bfloat16), (2000, 500, torch.bfloat16),
                                       (1017, 1032, torch.float32), (800, 2056, torch.bfloat16), (1020, 1536, torch.float32)])
def test_sums_of_fewer_than_256_workgroups(T, n, dtype):
    """25 to 250 rows of partial sums, which no multiple of 16 divides."""
    dY, H, gain = draw((T, n), 5, dtype, 0.3, 0.05), draw((T, n), 6, dtype, 1.5, 0.4), draw(n, 1, torch.float32, 0.2, 1.0)
    mean, rstd = stats(H, "layer")
    check_backward(dY, H, gain, mean, rstd, "layer", None, *gpu_backward(dY, H, gain, mean, rstd, "layer"))


@pytest.mark.parametrize("T,n,dtype", [(1024, 64, torch.bfloat16), (4099, 128, torch.float32), (4100, 512, torch.bfloat16),
                                       (3001, 1000, torch.bfloat16), (2600, 2056, torch.float32), (1500, 4096, torch.bfloat16),
                                       (1100, 5461, torch.bfloat16), (1030, 16385, torch.bfloat16), (2000, 1293, torch.float32),
                                       (1500, 2055, torch.bfloat16), (900, 4097, torch.bfloat16), (1200, 8193, torch.bfloat16),
                                       (500, 9001, torch.float32), (800, 16383, torch.float32)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_more_rows_than_workgroups_with_a_residual_branch(T, n, dtype, kind):
    """R and dR of the second row of a turn and after, and of the two kernels' path, against 64 bits."""
    gain, bias = draw(n, 1, torch.float32, 0.2, 1.0), draw(n, 2, torch.float32, 0.2)
    X, R = draw((T, n), 3, dtype, 1.5, 0.4), draw((T, n), 4, dtype)
    Y, H, mean, rstd = nan((T, n), dtype), nan((T, n), dtype), nan((T,)), nan((T,))
    grass.norm_forward(X, gain, bias, EPS, Y, KINDS[kind], R=R, H=H, mean=mean, rstd=rstd)
    check_forward(X, R, gain, bias, kind, Y, H, mean if kind == "layer" else None, rstd)
    dY, dR = draw((T, n), 5, dtype, 0.3, 0.05), draw((T, n), 7, dtype, 0.3)
    got = gpu_backward(dY, H, gain, mean, rstd, kind, dR)
    check_backward(dY, H, gain, mean if kind == "layer" else None, rstd, kind, dR, *got)


def streamed_bytes():
    """From so many bytes on accesses carry the streaming hint and the forward pass has more workgroups."""
    with open(os.path.join(os.path.dirname(__file__), "..", "paper_2406_17660_amd", "csrc", "elem.hpp")) as f:
        return float(re.search(r"kStreamed = ([0-9.]+) \* \(1 << 20\);", f.read()).group(1)) * (1 << 20)


STREAMED = [(64, torch.float32, 0, 3), (100, torch.bfloat16, 0, 3), (128, torch.bfloat16, 0, 3), (250, torch.bfloat16, 0, 1),
            (256, torch.bfloat16, 0, 3), (500, torch.bfloat16, 0, 1), (512, torch.bfloat16, 0, 2), (512, torch.float32, 8, 1),
            (601, torch.float32, 0, 1), (1000, torch.bfloat16, 0, 1), (1293, torch.bfloat16, 3, 1), (1536, torch.bfloat16, 0, 1),
            (2056, torch.bfloat16, 0, 1), (2601, torch.float32, 0, 1), (4096, torch.bfloat16, 0, 3), (4096, torch.float32, 0, 1),
            (4200, torch.bfloat16, 0, 1), (5461, torch.bfloat16, 0, 1), (5461, torch.float32, 1, 1), (8200, torch.bfloat16, 0, 1),
            (12289, torch.float32, 0, 1), (16384, torch.bfloat16, 0, 1), (16384, torch.float32, 0, 1)]


def streamed_rows(n, dtype, arrays, times):
    """Rows just beyond the limit, so many times over, whose last turn is partly filled."""
    size = n * dtype.itemsize * arrays
    T = int(times * streamed_bytes() // size) + 37
    assert T * size > streamed_bytes()
    return T


def rows_of(T, n, seed, dtype, more, scale=1.0, shift=0.0):
    values = draw((T, n), seed, dtype, scale, shift)
    return padded(values, n + more, 1)[0] if more else values


@pytest.mark.parametrize("n,dtype,more,times", STREAMED)
@pytest.mark.parametrize("add", [False, True])
def test_forward_of_more_than_the_cache_holds(n, dtype, more, times, add):
    """Against the formulas in 64 bits, with the bounds of check_forward."""
    T, layer = streamed_rows(n, dtype, 4 if add else 2, times), n % 3 != 0
    gain, bias = draw(n, 1, torch.float32, 0.2, 1.0), draw(n, 2, torch.float32, 0.2)
    X, R = rows_of(T, n, 3, dtype, more, 1.5, 0.4), rows_of(T, n, 4, dtype, more) if add else None
    Y, H = nan((T, n + more), dtype)[:, :n], nan((T, n + more), dtype)[:, :n] if add else None
    mean, rstd = nan((T,)), nan((T,))
    grass.norm_forward(X, gain, bias, EPS, Y, grass.NORM_LAYER if layer else grass.NORM_RMS, R=R, H=H, mean=mean, rstd=rstd)
    for a in range(0, T, max(1, (1 << 24) // n)):
        at = slice(a, a + max(1, (1 << 24) // n))
        h = X[at]
        if add:
            h = (h.float() + R[at].float()).to(dtype)
            assert torch.equal(H[at], h)
        h = h.double()
        size = h.abs().mean(1, keepdim=True)
        mu = h.mean(1, keepdim=True) if layer else torch.zeros_like(size)
        d = h - mu
        rs = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        y = d * rs * gain.double() + bias.double()
        assert ((Y[at].double() - y).abs() <= half(dtype) * y.abs() * (1 + FP32) +
                FP32 * (size * rs * gain.double().abs() + y.abs() + bias.double().abs())).all()
        if layer:
            assert ((mean[at].double() - mu[:, 0]).abs() <= FP32 * size[:, 0]).all()
        assert ((rstd[at].double() - rs[:, 0]).abs() <= (FP32 + (FP32 * size * rs)[:, 0] ** 2) * rs[:, 0]).all()
    if more:
        assert int((~torch.isnan(Y.as_strided((T - 1, more), (n + more, 1), n).float())).sum()) == 0


@pytest.mark.parametrize("n,dtype,more,times", STREAMED)
@pytest.mark.parametrize("add", [False, True])
def test_backward_of_more_than_the_cache_holds(n, dtype, more, times, add):
    """Against the formulas in 64 bits, with the bounds of check_backward."""
    T, layer = streamed_rows(n, dtype, 4 if add else 3, 1), n % 3 != 0
    gain = draw(n, 1, torch.float32, 0.2, 1.0)
    dY, H = rows_of(T, n, 5, dtype, more, 0.3, 0.05), rows_of(T, n, 6, dtype, more, 1.5, 0.4)
    dR = rows_of(T, n, 7, dtype, more, 0.3) if add else None
    mean = H.double().mean(1).float() if layer else None
    h = H.double() - mean.double()[:, None] if layer else H.double()
    rstd = (1.0 / torch.sqrt((h * h).mean(1) + EPS)).float()
    dX = nan((T, n + more), dtype)[:, :n]
    _, dgain, dbias = gpu_backward(dY, H, gain, mean, rstd, "layer" if layer else "rms", dR, dX)
    sums = torch.zeros((4, n), dtype=torch.float64, device=DEV)
    for a in range(0, T, max(1, (1 << 24) // n)):
        at = slice(a, a + max(1, (1 << 24) // n))
        dy, rs = dY[at].double(), rstd[at].double()[:, None]
        xh = h[at] * rs
        z = dy * gain.double()
        dx = z - xh * (z * xh).mean(1, keepdim=True)
        if layer:
            dx = dx - z.mean(1, keepdim=True)
        dx = dx * rs
        size = rs * (z.abs() + z.abs().mean(1, keepdim=True) + xh.abs() * (z * xh).abs().mean(1, keepdim=True))
        if add:
            dx, size = dx + dR[at].double(), size + dR[at].double().abs()
        assert ((dX[at].double() - dx).abs() <= half(dtype) * dx.abs() * (1 + FP32) + FP32 * size).all()
        for k, term in enumerate((dy * xh, dy, (dy * xh).abs(), dy.abs())):
            sums[k] += term.sum(0)
    for got, want, size in ((dgain, sums[0], sums[2]), (dbias, sums[1], sums[3])):
        assert ((got.double() - want).abs() <= depth(T) * 2.0 ** -24 * size).all()
    if more:
        assert int((~torch.isnan(dX.as_strided((T - 1, more), (n + more, 1), n).float())).sum()) == 0
