"""grass_embed_forward and grass_embed_backward against the same formulas in 64 bits.

Tolerances.  The lookup is one fp32 product, rounded once to its type: half a step, finfo.eps / 2, of either.  A sum
over c rows in any order is off by at most c half steps of fp32 of the sum of its magnitudes (c - 1 additions
and the product with the scale); adding to what is there takes one more of the result's magnitudes, and the result is
rounded once to its type."""
import numpy as np
import pytest
import torch

import ends_ref
from gpu_util import DEV, to_f64
from paper_2406_17660_amd import grass

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def draw(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def whole(shape, seed, most):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(most, shape, generator=g, device=DEV)


def padded(t, ld, offset):
    """The values of t in rows ld elements apart, the first `offset` elements behind the base; NaN around them."""
    T, n = t.shape
    flat = torch.full((offset + T * ld + 8,), float("nan"), dtype=t.dtype, device=DEV)
    view = flat[offset:offset + T * ld].view(T, ld)[:, :n]
    view.copy_(t)
    return view, flat


def nan(shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def half(dtype):
    return torch.finfo(dtype).eps / 2


def zipf(T, V, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    weight = (1.0 / (torch.arange(V, device=DEV, dtype=torch.float64) + 2.7)).cumsum(0)
    rank = torch.searchsorted(weight, torch.rand(T, generator=g, device=DEV, dtype=torch.float64) * weight[-1])
    return torch.randperm(V, generator=g, device=DEV)[rank.clamp(max=V - 1)]


# ---------------------------------------------------------------------------------- lookup
def check_lookup(E, ids, scale, Y):
    want = ends_ref.embed_forward(to_f64(E), ids.cpu().numpy().astype(np.int64), scale)
    assert (np.abs(to_f64(Y) - want) <= (U + half(Y.dtype) * (1 + U)) * np.abs(want)).all()


WIDTHS = [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 31, 40, 64, 65, 100, 127, 512, 513, 1000, 1293, 2048, 4096, 5461, 8200, 16384, 20001]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("edt,ydt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_lookup(n, edt, ydt):
    V, T = 37, (1, 2, 7, 65, 300)[n % 5]
    E, ids = draw((V, n), 1, edt), whole((T,), 2, V).to((torch.int32, torch.int64)[n % 2])
    if T > 4:
        ids[1], ids[3] = -1, V
    Y = nan((T, n), ydt)
    scale = 1.0 if n % 3 else 0.37
    grass.embed_forward(E, ids, Y, scale)
    check_lookup(E, ids, float(np.float32(scale)), Y)
    if scale == 1.0 and edt == ydt:
        there = (ids >= 0) & (ids < V)
        assert torch.equal(Y[there], E[ids[there].long()])


@pytest.mark.parametrize("edt,ydt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,more,offset", [(1, 1, 1), (5, 1, 1), (100, 3, 1), (512, 8, 8), (513, 2, 3), (4096, 5, 7)])
def test_lookup_rows_in_any_position(n, more, offset, edt, ydt):
    V, T = 21, 30
    E, ids = draw((V, n), 1, edt), whole((T + 1,), 2, V)[1:]
    vE, _ = padded(E, n + more, offset)
    vY, fY = padded(nan((T, n), ydt), n + more + 1, offset + 1)
    grass.embed_forward(vE, ids, vY, 2.5)
    check_lookup(E, ids, 2.5, vY)
    assert int((~torch.isnan(fY.float())).sum()) == vY.numel()


def test_token_numbers_of_64_bits_are_not_cut():
    E = draw((50, 24), 1, F32)
    ids = torch.tensor([3, (1 << 32) + 3, -(1 << 32) + 3, 1 << 62, -(1 << 63), 49, 50, -1], device=DEV)
    Y = nan((8, 24), F32)
    grass.embed_forward(E, ids, Y)
    assert torch.equal(Y[0], E[3]) and torch.equal(Y[5], E[49]) and not Y[[1, 2, 3, 4, 6, 7]].any()
    dE = nan((50, 24), F32)
    dY = draw((8, 24), 2, F32)
    backward(dY, ids, dE)
    assert torch.equal(dE[3], dY[0]) and torch.equal(dE[49], dY[5]) and int((dE != 0).any(1).sum()) == 2


def test_lookup_values_that_are_not_finite_stay_in_their_rows():
    E = draw((5, 20), 1, BF16)
    E[1, 3], E[2, 4], E[2, 5] = float("nan"), float("inf"), float("-inf")
    ids = torch.tensor([0, 1, 2, 3, -1], device=DEV)
    Y = nan((5, 20), F32)
    grass.embed_forward(E, ids, Y, 2.0)
    assert torch.equal(Y[:4].nan_to_num(7.0), (E[:4].float() * 2).nan_to_num(7.0)) and not Y[4].any()


def test_lookup_of_more_rows_than_a_grid():
    V, T, n = 19, 1300000, 3
    E, ids = draw((V, n), 1, BF16), whole((T,), 2, V)
    Y = nan((T, n), BF16)
    grass.embed_forward(E, ids, Y)
    assert torch.equal(Y, E[ids])


@pytest.mark.parametrize("far", ["E", "Y"])
def test_lookup_offsets_beyond_32_bits(far):
    ld, n = (1 << 30) + 8, 40  # elements between rows, 2 GB of bf16
    V, T = 4, 4
    E, ids = draw((V, n), 1, BF16), torch.tensor([3, 0, 2, 3], device=DEV)
    Y = nan((T, n), BF16)
    room = torch.empty(3 * ld + n, dtype=BF16, device=DEV)
    view = torch.as_strided(room, (4, n), (ld, 1))
    if far == "E":
        view.copy_(E)
        grass.embed_forward(view, ids, Y)
        assert torch.equal(Y, E[ids])
    else:
        view.zero_()
        grass.embed_forward(E, ids, view)
        assert torch.equal(view, E[ids])


# -------------------------------------------------------------------------------- gradient
def backward(dY, ids, dE, scale=1.0, accumulate=False):
    (T, n), V = dY.shape, dE.shape[0]
    need = grass.embed_backward_workspace(T, V, n)
    room = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    grass.embed_backward(dY, ids, dE, room[:need] if need else None, scale, accumulate)
    assert bool((room[need:] == 0xFF).all()), "nothing behind the workspace is written"
    return dE


def check_gradient(dY, ids, dE, scale, was=None):
    want, size, count = ends_ref.embed_backward(to_f64(dY), ids.cpu().numpy().astype(np.int64), dE.shape[0], scale)
    if was is not None:
        want, size = want + to_f64(was), size + np.abs(to_f64(was))
        untouched = torch.from_numpy(count == 0).to(dE.device)
        assert torch.equal(dE[untouched], was[untouched])
    else:
        assert not to_f64(dE)[count == 0].any()
    off = (count[:, None] + 2) * U * size
    assert (np.abs(to_f64(dE) - want) <= off + half(dE.dtype) * (np.abs(want) + off) * (dE.dtype == BF16)).all()


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("dt,gdt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_gradient(n, dt, gdt):
    V, T = (37, 300)[n % 2], (1, 200, 65, 300, 1000)[n % 5]
    dY, ids = draw((T, n), 3, dt), zipf(T, V, 4).to((torch.int32, torch.int64)[n % 2])
    if T > 4:
        ids[1], ids[3] = -1, V
    was = draw((V, n), 5, gdt) if n % 3 == 0 else None
    dE = nan((V, n), gdt) if was is None else was.clone()
    backward(dY, ids, dE, 0.5 if n % 4 else 1.7, was is not None)
    check_gradient(dY, ids, dE, 0.5 if n % 4 else float(np.float32(1.7)), was)


# tokens and vocabularies about the sizes where sorting and summing go another way
SIZES = [(1, 1), (1, 100000), (31, 3), (32, 1), (33, 1), (63, 2), (64, 64), (65, 70000), (127, 5), (128, 2), (129, 1), (255, 40), (256, 3), (256, 50000), (257, 40), (1023, 255), (1024, 256),
         (1025, 257), (2047, 511), (2048, 512), (2049, 513), (4095, 32000), (4096, 9), (4097, 65536), (8191, 65537), (8192, 1000),
         (8193, 4096), (16385, 262143), (16384, 262144), (20000, 262145), (30001, 2), (65536, 32000), (100003, 300)]


@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("how", ["zipf", "uniform", "one", "runs"])
def test_gradient_of_many_tokens(T, V, how):
    """Also one token alone in all places, and tokens in falling runs."""
    n, dt = 24, BF16
    ids = {"zipf": lambda: zipf(T, V, 6), "uniform": lambda: whole((T,), 6, V), "one": lambda: torch.full((T,), V // 2, device=DEV),
           "runs": lambda: V - 1 - torch.arange(T, device=DEV) // 37 % V}[how]()
    if T > 60:
        ids[::17] = -1
    dY = draw((T, n), 7, dt)
    dE = backward(dY, ids, nan((V, n), F32))
    check_gradient(dY, ids, dE, 1.0)
    assert torch.equal(backward(dY, ids, nan((V, n), F32)), dE), "equal calls give equal bits"
    was = draw((V, n), 8, F32)
    check_gradient(dY, ids, backward(dY, ids, was.clone(), 0.25, True), 0.25, was)


@pytest.mark.parametrize("dt,gdt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,more,offset", [(1, 1, 1), (5, 1, 1), (100, 3, 1), (512, 8, 8), (513, 2, 3), (1030, 5, 7)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_rows_in_any_position(n, more, offset, dt, gdt, accumulate):
    V, T = 13, (200, 400)[offset % 2]
    dY, ids = draw((T, n), 3, dt), zipf(T, V - 2, 4)
    vY, _ = padded(dY, n + more, offset)
    was = draw((V, n), 5, gdt)
    vE, fE = padded(was if accumulate else nan((V, n), gdt), n + more + 1, offset + 1)
    backward(vY, ids, vE, 1.5, accumulate)
    check_gradient(dY, ids, vE, 1.5, was if accumulate else None)
    assert int((~torch.isnan(fE.float())).sum()) == vE.numel()


@pytest.mark.parametrize("V", [5, 40000])
def test_gradient_of_padding_alone_and_of_no_tokens(V):
    n = 50
    for ids in (torch.full((90,), -100, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV)):
        dY = nan((len(ids), n), BF16)
        assert not backward(dY, ids, nan((V, n), BF16)).any()
        was = nan((V, n), F32)
        assert bool(torch.isnan(backward(dY, ids, was, accumulate=True)).all())


def test_gradient_values_that_are_not_finite_stay_in_their_rows():
    """Rows of padding are not read, and a NaN or an infinity reaches its own token's row and column alone."""
    T, V, n = 400, 30, 64
    ids, dY = zipf(T, V, 9), draw((T, n), 10, F32)
    ids[5], ids[77] = -1, V
    dY[5], dY[77] = float("nan"), float("inf")
    dY[9, 3], dY[200, 60] = float("nan"), float("inf")
    dE = backward(dY, ids, nan((V, n), F32))
    bad = ~torch.isfinite(dE)
    assert int(bad.sum()) == 2 and bool(bad[ids[9], 3]) and bool(bad[ids[200], 60])


@pytest.mark.parametrize("far", ["dY", "dE"])
def test_gradient_offsets_beyond_32_bits(far):
    ld, n = (1 << 30) + 8, 40
    ids = torch.tensor([3, 0, 2, 3], device=DEV)
    dY = draw((4, n), 1, BF16)
    room = torch.empty(3 * ld + n, dtype=BF16, device=DEV)
    view = torch.as_strided(room, (4, n), (ld, 1))
    if far == "dY":
        view.copy_(dY)
        check_gradient(dY, ids, backward(view, ids, nan((4, n), F32)), 1.0)
    else:
        view.fill_(float("nan"))
        check_gradient(dY, ids, backward(dY, ids, view), 1.0)


def test_gradient_of_a_long_batch_and_wide_rows():
    """Sums of up to thousands of rows, split over workgroups, at a width that several of them share."""
    T, V, n = 40000, 500, 3001
    dY, ids = draw((T, n), 1, BF16), zipf(T, V, 2)
    dE = backward(dY, ids, nan((V, n), F32), 0.125)
    want, size, count = torch.zeros((V, n), dtype=torch.float64, device=DEV), torch.zeros((V, n), dtype=torch.float64, device=DEV), ids.bincount(minlength=V)
    for a in range(0, T, 8000):
        part = dY[a:a + 8000].double() * 0.125
        want.index_add_(0, ids[a:a + 8000], part)
        size.index_add_(0, ids[a:a + 8000], part.abs())
    assert bool(((dE.double() - want).abs() <= (count.view(-1, 1) + 2) * U * size).all())


@pytest.mark.parametrize("T,V", [(530000, 700), (1100003, 70001), (600000, 1)])
def test_gradient_of_more_tokens_than_workgroups_sort_at_a_time(T, V):
    n = 5
    dY, ids = draw((T, n), 1, F32), zipf(T, V, 2)
    ids[::11] = -1
    dE = backward(dY, ids, nan((V, n), F32))
    row = torch.where(ids < 0, V, ids)
    want, size = (torch.zeros((V + 1, n), dtype=torch.float64, device=DEV).index_add_(0, row, x.double())[:V] for x in (dY, dY.abs()))
    count = row.bincount(minlength=V + 1)[:V].view(-1, 1)
    assert bool(((dE.double() - want).abs() <= (count + 2) * U * size).all())
    assert torch.equal(backward(dY, ids, nan((V, n), F32)), dE)


def test_workspace_serves_shorter_batches():
    V, n = 32000, 512
    sizes = [grass.embed_backward_workspace(T, V, n) for T in (0, 1, 100, 2047, 4096, 32000, 32736, 32737, 65536, 524288, 524289, 2000000)]
    assert sizes == sorted(sizes)
    ws = grass.workspace(grass.embed_backward_workspace(40000, V, n))
    for T in (32736, 5, 40000, 1000):
        dY, ids = draw((T, n), T, BF16), zipf(T, V, 3)
        dE = grass.embed_backward(dY, ids, nan((V, n), F32), ws)
        assert torch.equal(dE, backward(dY, ids, nan((V, n), F32)))


# ------------------------------------------------------------------- streams, graphs, checks
@pytest.mark.parametrize("T,V,n", [(700, 90, 136), (40000, 3000, 136)])
def test_on_another_stream_and_in_a_graph(T, V, n):
    E, dY = draw((V, n), 1, BF16), draw((T, n), 2, BF16)
    ids, ids2 = zipf(T, V, 3), whole((T,), 4, V)
    Y, dE, was = nan((T, n), BF16), nan((V, n), F32), draw((V, n), 5, F32)
    ws = grass.workspace(grass.embed_backward_workspace(T, V, n))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    held = ids.clone()
    with torch.cuda.stream(side):
        grass.embed_forward(E, held, Y)
        grass.embed_backward(dY, held, dE, ws)
    torch.cuda.current_stream().wait_stream(side)
    first = dE.clone()
    check_lookup(E, ids, 1.0, Y)
    check_gradient(dY, ids, dE, 1.0)
    graph = torch.cuda.CUDAGraph()
    more = was.clone()
    with torch.cuda.graph(graph):
        grass.embed_forward(E, held, Y)
        grass.embed_backward(dY, held, dE, ws)
        grass.embed_backward(dY, held, more, ws, 0.5, accumulate=True)
    for turn in range(4):
        now = (ids, ids2)[turn % 2]
        held.copy_(now)
        more.copy_(was)
        Y.fill_(float("nan"))
        dE.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check_lookup(E, now, 1.0, Y)
        check_gradient(dY, now, dE, 1.0)
        check_gradient(dY, now, more, 0.5, was)
        assert torch.equal(backward(dY, now, nan((V, n), F32)), dE) and (turn % 2 or torch.equal(dE, first))


def test_binding_refuses():
    E, ids, Y = draw((8, 6), 1, F32), whole((4,), 2, 8), nan((4, 6), F32)
    bad = [(E.t(), ids, nan((4, 8), F32)), (E, ids.float(), Y), (E, ids[:3], Y), (E, ids, nan((4, 5), F32)), (E.half(), ids, Y),
           (E, whole((8,), 2, 8)[::2], Y), (E, ids, nan((1, 12), F32)[:, ::2]), (E, ids.cpu(), Y)]
    for e, i, y in bad:
        with pytest.raises((AssertionError, TypeError)):
            grass.embed_forward(e, i, y)
        with pytest.raises((AssertionError, TypeError)):
            grass.embed_backward(y, i, e, grass.workspace(1 << 16))
