"""Forms of the kernels at a model's two ends that ordinary small batches do not reach."""
import pytest
import torch

from gpu_util import DEV
from paper_2406_17660_amd import grass
from test_gpu_logp import backward, forward, special

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


def same_bits(a, b):
    """Equal, a NaN to a NaN too."""
    return a.dtype == b.dtype and torch.equal(a.view(torch.int16 if a.dtype == BF16 else torch.int32),
                                              b.view(torch.int16 if b.dtype == BF16 else torch.int32))


def embed_backward(dY, ids, dE, scale=1.0, accumulate=False):
    ws = grass.workspace(grass.embed_backward_workspace(dY.shape[0], dE.shape[0], dE.shape[1]))
    return grass.embed_backward(dY, ids, dE, ws, scale, accumulate)


@pytest.mark.parametrize("T,V", [(T, V) for T in (4000, 20000, 70000, 700000) for V in (3, 300, 600)])
def test_places_are_counted_whichever_lane_leads(T, V):
    """A token's first place among the 64 that a wavefront counts at a time is in another lane each time.  Rows of small whole
    numbers: their sums, below 2^24, are exact in fp32 in any order."""
    i = torch.arange(T, device=DEV)
    ids = (i + i // 64) % V
    dY = torch.stack([torch.ones_like(i), i % 7 - 3, i // 64 % 5], 1).to(BF16)
    want = torch.zeros((V, 3), dtype=torch.float64, device=DEV).index_add_(0, ids, dY.double())
    dE = embed_backward(dY, ids, torch.full((V, 3), float("nan"), device=DEV))
    assert torch.equal(dE.double(), want)


# ----------------------------------------------------------- workgroups that take several turns
@pytest.fixture(params=[1, 3])
def few_blocks(request):
    """In a call of it, kernels walk over rows and pieces in one workgroup or three.  Each shape below has work for four and more;
    equal calls give equal bits on any number of them."""
    def within(call):
        grass.set_test_option(grass.TEST_MOST_BLOCKS, request.param)
        try:
            return call()
        finally:
            grass.set_test_option(grass.TEST_MOST_BLOCKS, 0)
    return within


# one V in each shape of the forward pass (64 threads and 1, 2, 4, 8 vectors; 256 and 4, 8; 512 and 5, 8; rows in parts), for bf16 / fp32
@pytest.mark.parametrize("dtype,V", [(BF16, v) for v in (1, 7, 300, 512, 1000, 2048, 4001, 8192, 16000, 20480, 32768, 32769, 140003)] +
                         [(F32, v) for v in (3, 256, 500, 1024, 2001, 4096, 8000, 10240, 16384, 16385, 70001)])
@pytest.mark.parametrize("top", [0, 20])
def test_log_probabilities_in_few_workgroups(few_blocks, dtype, V, top):
    """Rows whose lists of alternatives overflow, rows of NaN, masked and ordinary ones behind each other in a workgroup."""
    if V < 4:
        x = draw((60, V), 1, dtype)
        x[::7] = float("-inf")
    else:
        _, x = special(V, dtype, V)
        x = x[torch.randperm(len(x), generator=torch.Generator().manual_seed(V)).to(DEV).repeat(3)]
    T, top = len(x), min(top, V)
    targets = whole((T,), 2, V)
    targets[5] = -100
    want, got = forward(x, targets, top, 0.5), few_blocks(lambda: forward(x, targets, top, 0.5))
    for name in want:
        assert (want[name] is None and got[name] is None) or same_bits(got[name], want[name]), name
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    dlogp[::5], dH[::5] = 0.0, 0.0
    for H, d in ((None, None), (want["entropy"], dH)):
        f = lambda: backward(x, targets, want["rmax"], want["rlog"], dlogp, 0.5, H, d)  # noqa: E731
        assert same_bits(few_blocks(f), f())


@pytest.mark.parametrize("edt,ydt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("T,n", [(70000, 1), (9000, 5), (3000, 24), (70, 1293), (40, 4096), (3, 70001)])
def test_lookup_in_few_workgroups(few_blocks, T, n, edt, ydt):
    E, ids = draw((37, n), 1, edt), whole((T,), 2, 39) - 1  # (-1 and 37: padding)
    for scale in (1.0, 0.37):
        want, got = (f(lambda: grass.embed_forward(E, ids, torch.full((T, n), float("nan"), dtype=ydt, device=DEV), scale))
                     for f in (lambda g: g(), few_blocks))
        assert same_bits(got, want)


# up to 256 places; one-kernel ordering, pieces of 8 and of 32; radix sort; few rows and many that no token has
@pytest.mark.parametrize("T,V,n", [(200, 7, 24), (256, 5000, 24), (256, 9, 3001), (300, 70, 24), (5000, 9000, 3), (5000, 40, 1100), (20000, 300, 600),
                                   (40000, 3000, 130), (70000, 20, 520)])
@pytest.mark.parametrize("dt,gdt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_the_embedding_in_few_workgroups(few_blocks, T, V, n, dt, gdt, accumulate):
    dY, ids = draw((T, n), 1, dt), whole((T,), 2, V + 2) - 1
    ids[T // 3:T // 2] = V // 2  # a frequent one
    was = draw((V, n), 3, gdt) if accumulate else torch.full((V, n), float("nan"), dtype=gdt, device=DEV)
    want, got = (f(lambda: embed_backward(dY, ids, was.clone(), 0.5, accumulate)) for f in (lambda g: g(), few_blocks))
    assert bool(torch.isfinite(want.float()).all()) and same_bits(got, want)


# ---------------------------------------------------------------- large calls: the streaming hint
# Forward and backward passes carry it from 128 MiB on, the gradient of the embedding also where dE is above 32 MiB.  Such arrays are
# compared on the card, in 64 bits, some rows at a time; the tolerances are those of the tests of each operator.
STREAMED = 128 << 20


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype == BF16 else 0.0


def rows_at_a_time(T, n):
    step = max(1, (1 << 25) // n)
    return [slice(a, min(a + step, T)) for a in range(0, T, step)]


def check_statistics(x, targets, scale, out):
    """As derived for the forward pass: with E = entropy - rlog the sum of exponentials is off by SUM, log p by SUM + 4 U (|d| + rlog), the
    entropy by SUM (1 + E) + 4 U (rlog + E)."""
    V = x.shape[1]
    for r in rows_at_a_time(*x.shape):
        z = x[r].double()
        m = z.amax(1, keepdim=True)
        d = (z - m) * scale
        rlog = d.exp().sum(1).log()
        E = -((d - rlog.view(-1, 1)).exp() * d).sum(1)
        SUM = (264 + 3 * E + rlog) * U
        given = d.gather(1, targets[r].view(-1, 1))[:, 0]
        assert torch.equal(out["rmax"][r].double(), m[:, 0])
        assert bool(((out["rlog"][r].double() - rlog).abs() <= SUM).all())
        assert bool(((out["logp"][r].double() - (given - rlog)).abs() <= SUM + 4 * U * (given.abs() + rlog)).all())
        if out["entropy"] is not None:
            assert bool(((out["entropy"][r].double() - (rlog + E)).abs() <= SUM * (1 + E) + 4 * U * (rlog + E)).all())
        if out["top_idx"] is not None:
            order = (x[r].float() + 0.0).view(torch.int32)
            order = torch.where(order < 0, order ^ 0x7FFFFFFF, order).long() * (1 << 32) - torch.arange(V, device=DEV)
            idx = torch.topk(order, out["top_idx"].shape[1], dim=1).indices
            assert torch.equal(out["top_idx"][r].long(), idx)
            best = d.gather(1, idx)
            off = SUM.view(-1, 1) + 4 * U * (best.abs() + rlog.view(-1, 1))
            assert bool(((out["top_logp"][r].double() - (best - rlog.view(-1, 1))).abs() <= off).all())


def check_gradient_of_logits(x, targets, scale, out, dlogp, dentropy, dx):
    """With rmax and rlog as they are given, p is off by (4 (|d| + rlog) + 8) U of itself."""
    for r in rows_at_a_time(*x.shape):
        col = lambda v: v[r].double().view(-1, 1)  # noqa: E731
        rlog, H, g = col(out["rlog"]), col(out["entropy"]), col(dlogp)
        h = torch.zeros_like(g) if dentropy is None else col(dentropy)
        d = (x[r].double() - col(out["rmax"])) * scale
        l = d - rlog
        p = l.exp()
        want = -p * (g + h * (l + H))
        arg = d.abs() + rlog
        rel = (4 * arg + 8) * U
        size = p * (g.abs() * (rel + 2 * U) + h.abs() * ((l.abs() + H) * (rel + 4 * U) + 4 * U * (arg + l.abs() + H)))
        j = targets[r].view(-1, 1)
        want.scatter_add_(1, j, g)
        size.scatter_add_(1, j, 4 * U * g.abs())
        want, size = want * scale, size * scale
        off = size + 2 * U * want.abs() + half_step(dx.dtype) * (want.abs() + size) + 2.0 ** -120 * (1 + g.abs() + h.abs())
        assert bool(((dx[r].double() - want).abs() <= off).all())


# one V in each shape, as above, and enough rows
@pytest.mark.parametrize("dtype,V", [(BF16, v) for v in (100, 300, 1000, 2048, 4001, 8192, 16000, 20480, 32000, 50001, 140003)] +
                         [(F32, v) for v in (50, 256, 500, 1024, 2001, 4096, 8000, 10240, 16384, 50001, 70001)])
def test_log_probabilities_of_large_calls(dtype, V):
    T = STREAMED // (V * dtype.itemsize) + 17
    x, targets = draw((T, V), 1, dtype, 2.0), whole((T,), 2, V)
    dlogp, dH = draw((T,), 3, F32), draw((T,), 4, F32)
    for top, entropy in ((9, True), (9, False), (0, False), (0, True)):
        out = forward(x, targets, top, 0.5, entropy=entropy)
        check_statistics(x, targets, 0.5, out)
    for d in (None, dH):
        dx = backward(x, targets, out["rmax"], out["rlog"], dlogp, 0.5, None if d is None else out["entropy"], d)
        check_gradient_of_logits(x, targets, 0.5, out, dlogp, d, dx)
    dlogp[::3], dH[::3], targets[1::3] = 0.0, 0.0, -1  # rows that are not read
    x[::3] = float("nan")
    again = backward(x, targets, out["rmax"], out["rlog"], dlogp, 0.5, out["entropy"], dH)
    assert not again[::3].any() and torch.equal(again[2::3], dx[2::3])


@pytest.mark.parametrize("edt,ydt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("T,n", [(1100000, 70), (40000, 4096), (20001, 5461)])
@pytest.mark.parametrize("scale", [1.0, 0.37])
def test_lookup_of_large_calls(T, n, edt, ydt, scale):
    """One fp32 product, rounded once to its type; with a scale of one and one type the bits as they are."""
    V = 20000
    E, ids = draw((V, n), 1, edt), whole((T,), 2, V + 2) - 1
    Y = torch.full((T, n), float("nan"), dtype=ydt, device=DEV)
    assert Y.nbytes > STREAMED
    grass.embed_forward(E, ids, Y, scale)
    there = ((ids >= 0) & (ids < V)).view(-1, 1)
    exact = torch.tensor(scale, dtype=F32).double().item()
    for r in rows_at_a_time(T, n):
        want = E[ids[r].clamp(0, V - 1)].double() * exact * there[r]
        if scale == 1.0 and edt == ydt:
            assert torch.equal(Y[r].double(), want)
        else:
            assert bool(((Y[r].double() - want).abs() <= (U + half_step(ydt) * (1 + U)) * want.abs()).all())


# dY and dE streamed, in pieces of 32; dE alone, in pieces of 32 and of 8; dE of a few places
@pytest.mark.parametrize("T,V,n", [(40000, 20000, 2048), (40000, 32000, 640), (5000, 9000, 2048), (100, 9000, 2048), (40011, 19001, 2051),
                                   (5003, 9001, 2051), (101, 9001, 2051)])
@pytest.mark.parametrize("dt,gdt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_the_embedding_of_large_calls(T, V, n, dt, gdt, accumulate):
    """Sums of c rows: (c + 2) half steps of fp32 of the magnitudes, and one rounding to the type."""
    dY, ids = draw((T, n), 1, dt), (torch.rand(T, device=DEV, generator=torch.Generator(DEV).manual_seed(2)) ** 3 * (V + 1)).long() - 1
    ids[T // 4:T // 3] = V // 2
    was = draw((V, n), 3, gdt) if accumulate else torch.full((V, n), float("nan"), dtype=gdt, device=DEV)
    dE = embed_backward(dY, ids, was.clone(), 0.5, accumulate)
    assert dE.nbytes > 1 << 25
    row = torch.where((ids >= 0) & (ids < V), ids, V)
    count = row.bincount(minlength=V + 1)[:V].view(-1, 1)
    want, size = (torch.zeros((V + 1, n), dtype=torch.float64, device=DEV) for _ in range(2))
    for r in rows_at_a_time(T, n):
        want.index_add_(0, row[r], dY[r].double() * 0.5)
        size.index_add_(0, row[r], dY[r].double().abs() * 0.5)
    want, size = want[:V], size[:V]
    if accumulate:
        want, size = want + was.double(), size + was.double().abs()
        assert torch.equal(dE[count[:, 0] == 0], was[count[:, 0] == 0])
    off = (count + 2) * U * size
    assert bool(((dE.double() - want).abs() <= off + half_step(gdt) * (want.abs() + off)).all())


# the radix sort: chunks in registers, several passes, chunks read again; and the one-kernel ordering
@pytest.mark.parametrize("T,V", [(65536, 32000), (20000, 262145), (33000, 1), (600000, 700), (1000, 300), (30000, 9)])
def test_token_numbers_of_32_bits(T, V):
    """Rows of small whole numbers, whose sums are exact in any order; padding of either sign, the largest numbers among it."""
    ids = whole((T,), 1, V).int()
    ids[::13] = torch.tensor([-1, V, -100, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device=DEV).repeat(T)[:len(ids[::13])]
    dY = whole((T, 5), 2, 9).to(BF16) - 4
    there = (ids >= 0) & (ids < V)
    want = torch.zeros((V, 5), dtype=torch.float64, device=DEV).index_add_(0, ids[there].long(), dY[there].double())
    dE = embed_backward(dY, ids, torch.full((V, 5), float("nan"), device=DEV))
    assert torch.equal(dE.double(), want)
    assert torch.equal(embed_backward(dY, ids.long(), torch.full((V, 5), float("nan"), device=DEV)), dE)
