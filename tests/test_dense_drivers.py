"""What the drivers of the embedding, the norms and the log probabilities keep between their calls, and what they refuse
(CPU only: the library's calls are replaced by ones that accept, or refuse, whatever they are given)."""
import pytest
import torch

from paper_2406_17660_amd import grass
from paper_2406_17660_amd.dense import Embedding, NormLayer, TokenLoss

F32, BF16 = torch.float32, torch.bfloat16


class Refused(Exception):
    pass


@pytest.fixture
def library(monkeypatch):
    """The calls that were made, by name; those named in `refuse` raise."""
    class Calls(list):
        refuse = ()
    calls = Calls()

    def stand_in(name, result):
        def f(*args, **kw):
            if name in calls.refuse:
                raise Refused(name)
            calls.append(name)
            return args[result]
        monkeypatch.setattr(grass, name, f)
    for name, result in (("embed_forward", 2), ("embed_backward", 2), ("logp_forward", 2), ("logp_backward", 5), ("norm_forward", 4),
                         ("norm_backward", 5)):
        stand_in(name, result)
    return calls


def loss_and_batch():
    return TokenLoss(8, 12, F32, device="cpu"), torch.zeros(5, 12), torch.zeros(5, dtype=torch.int64), torch.zeros(5)


@pytest.mark.parametrize("how", ["by the library", "for its length"])
def test_no_gradient_after_a_refused_forward_pass_of_the_loss(library, how):
    """rmax and rlog are still those of the batch before: with the new logits they would give a wrong gradient."""
    loss, logits, targets, dlogp = loss_and_batch()
    loss.forward(logits, targets)
    if how == "by the library":
        library.refuse = ("logp_forward",)
        with pytest.raises(Refused):
            loss.forward(torch.ones(5, 12), targets)
    else:
        with pytest.raises(AssertionError):
            loss.forward(torch.ones(9, 12), torch.zeros(9, dtype=torch.int64))
    with pytest.raises(AssertionError):
        loss.backward(dlogp)
    assert "logp_backward" not in library
    library.refuse = ()
    loss.forward(logits, targets)
    assert loss.backward(dlogp) is logits


def test_a_refused_gradient_of_the_loss_leaves_the_logits_for_another(library):
    loss, logits, targets, dlogp = loss_and_batch()
    loss.forward(logits, targets)
    library.refuse = ("logp_backward",)
    with pytest.raises(Refused):
        loss.backward(dlogp)
    library.refuse = ()
    assert loss.backward(dlogp) is logits
    with pytest.raises(AssertionError):  # now they are written over
        loss.backward(dlogp)


@pytest.mark.parametrize("how", ["no pass", "by the library", "for its length"])
def test_no_gradient_of_the_embedding_without_a_forward_pass(library, how):
    layer, dY = Embedding(torch.zeros(12, 6), 8), torch.zeros(5, 6)
    if how != "no pass":
        layer.forward(torch.zeros(5, dtype=torch.int64))
        library.refuse = ("embed_forward",) if how == "by the library" else ()
        with pytest.raises((Refused, AssertionError)):
            layer.forward(torch.ones(9 if how == "for its length" else 5, dtype=torch.int64))
    with pytest.raises(AssertionError, match="forward pass"):
        layer.backward(dY)
    assert "embed_backward" not in library
    library.refuse = ()
    layer.forward(torch.zeros(5, dtype=torch.int64))
    assert layer.backward(dY) is layer.dE and layer.backward(dY, accumulate=True) is layer.dE


@pytest.mark.parametrize("dE", [torch.zeros(11, 6), torch.zeros(13, 6), torch.zeros(12, 5), torch.zeros(72), torch.zeros(1, 12, 6),
                                torch.zeros(12, 6, device="meta")])
def test_a_given_gradient_has_the_embeddings_shape_and_device(dE):
    """One of fewer rows would lose the tokens beyond them, which then count as padding."""
    with pytest.raises(AssertionError, match="gradient"):
        Embedding(torch.zeros(12, 6), 8, dE=dE)


def test_a_given_gradient_of_the_embedding_of_either_type_is_kept():
    for dtype in (F32, BF16):
        dE = torch.zeros((12, 6), dtype=dtype)
        assert Embedding(torch.zeros((12, 6), dtype=BF16), 8, dE=dE).parameters()[0][1] is dE
    with pytest.raises(TypeError):
        Embedding(torch.zeros(12, 6), 8, dE=torch.zeros(12, 6).half())


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32, torch.uint16])
def test_types_that_no_kernel_takes_are_refused_at_construction(dtype):
    """They would count as bf16, and fail, or find a workspace of another size, in the first call alone."""
    with pytest.raises(TypeError):
        TokenLoss(8, 12, dtype, device="cpu")
    with pytest.raises(TypeError):
        NormLayer(12, 8, dtype, device="cpu")
    for dtype in (F32, BF16):
        TokenLoss(8, 12, dtype, device="cpu"), NormLayer(12, 8, dtype, device="cpu")


@pytest.mark.parametrize("how", ["no pass", "by the library", "for its length"])
@pytest.mark.parametrize("residual", [False, True])
def test_no_gradient_of_the_norm_without_a_forward_pass(library, residual, how):
    """rstd (and mean) are still those of the batch before."""
    layer, dY = NormLayer(6, 8, F32, device="cpu"), torch.zeros(5, 6)
    if how != "no pass":
        layer.forward(torch.zeros(5, 6))
        library.refuse = ("norm_forward",) if how == "by the library" else ()
        X = torch.ones(9 if how == "for its length" else 5, 6)
        with pytest.raises((Refused, AssertionError)):
            layer.forward(X, R=X if residual else None)
    with pytest.raises(AssertionError, match="forward pass"):
        layer.backward(dY)
    assert "norm_backward" not in library
    library.refuse = ()
    X = torch.zeros(5, 6)
    layer.forward(X)
    assert layer.H is X and layer.backward(dY).shape == (5, 6)
