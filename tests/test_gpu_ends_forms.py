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
