"""Forms of the kernels at a model's two ends that ordinary small batches do not reach."""
import pytest
import torch

from gpu_util import DEV
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
