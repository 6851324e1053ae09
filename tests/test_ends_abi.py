"""What the embedding and the log probabilities refuse on the host, before anything is launched (CPU only)."""
import pytest
import torch

from paper_2406_17660_amd import grass

FAKE, ODD = 0x1000, 0x1001  # never dereferenced
OK, NULL, SHAPE, DTYPE, WS = grass.OK, grass.ERR_NULL, grass.ERR_SHAPE, grass.ERR_DTYPE, grass.ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


def call(f, names, values, **kw):
    assert set(kw) <= set(names)
    return f(*[kw.get(n, v) for n, v in zip(names, values)])


def embed_forward(**kw):
    return call(grass.lib().grass_embed_forward, "E edt V n lde ids idt T scale Y ydt ldy stream".split(),
                (FAKE, 1, 100, 64, 64, FAKE, 1, 8, 1.0, FAKE, 0, 64, None), **kw)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(E=None)), (NULL, dict(ids=None)), (NULL, dict(Y=None)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=BIG)), (SHAPE, dict(V=0)),
    (SHAPE, dict(V=BIG)), (SHAPE, dict(n=0)), (SHAPE, dict(n=BIG)), (SHAPE, dict(lde=63)), (SHAPE, dict(ldy=63)), (SHAPE, dict(scale=NAN)),
    (SHAPE, dict(scale=INF)), (SHAPE, dict(E=ODD)), (SHAPE, dict(Y=FAKE + 2)), (SHAPE, dict(ids=FAKE + 4)), (SHAPE, dict(idt=0, ids=FAKE + 2)),
    (DTYPE, dict(edt=2)), (DTYPE, dict(ydt=-1)), (DTYPE, dict(idt=2)), (OK, dict(T=0)), (OK, dict(T=0, E=None, Y=None, ids=None))])
def test_embed_forward_validation(want, kw):
    assert embed_forward(**kw) == want


def embed_backward(**kw):
    return call(grass.lib().grass_embed_backward,
                "dY dt lddy ids idt T V n scale accumulate dE gdt ldde ws ws_bytes stream".split(),
                (FAKE, 1, 64, FAKE, 1, 8, 100, 64, 1.0, 0, FAKE, 0, 64, FAKE, 1 << 40, None), **kw)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(dY=None)), (NULL, dict(ids=None)), (NULL, dict(dE=None)), (NULL, dict(dE=None, T=0)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=BIG)),
    (SHAPE, dict(V=0)), (SHAPE, dict(V=BIG)), (SHAPE, dict(n=0)), (SHAPE, dict(n=BIG)), (SHAPE, dict(lddy=63)), (SHAPE, dict(ldde=63)),
    (SHAPE, dict(scale=NAN)), (SHAPE, dict(scale=-INF)), (SHAPE, dict(dY=ODD)), (SHAPE, dict(dE=FAKE + 2)), (SHAPE, dict(ids=FAKE + 4)),
    (DTYPE, dict(dt=2)), (DTYPE, dict(gdt=7)), (DTYPE, dict(idt=-1)), (OK, dict(T=0, accumulate=1)),
    (OK, dict(T=0, accumulate=1, dY=None, ids=None))])
def test_embed_backward_validation(want, kw):
    assert embed_backward(**kw) == want


def test_embed_backward_workspace():
    q = grass.embed_backward_workspace
    assert q(-1, 4, 4) == q(4, 0, 4) == q(4, 4, 0) == q(BIG, 4, 4) == q(4, BIG, 4) == q(4, 4, BIG) == 0
    for T, V, n in ((1, 3, 5), (1000, 50, 64), (70000, 32000, 512), (5000, 300000, 1000)):
        need = q(T, V, n)
        kw = dict(T=T, V=V, n=n, lddy=n, ldde=n)
        if need:
            assert embed_backward(ws_bytes=need - 1, **kw) == embed_backward(ws=None, **kw) == embed_backward(ws=FAKE + 8, **kw) == WS


def logp_forward(**kw):
    return call(grass.lib().grass_logp_forward,
                "logits dt T V ldl targets idt scale logp entropy rmax rlog top top_logp top_idx ws ws_bytes stream".split(),
                (FAKE, 1, 8, 64, 64, FAKE, 1, 1.0, FAKE, FAKE, FAKE, FAKE, 5, FAKE, FAKE, FAKE, 1 << 40, None), **kw)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(logits=None)), (NULL, dict(targets=None)), (NULL, dict(logp=None)), (NULL, dict(top_logp=None)), (NULL, dict(top_idx=None)),
    (NULL, dict(top=0)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=BIG)), (SHAPE, dict(V=0)), (SHAPE, dict(V=BIG)), (SHAPE, dict(ldl=63)),
    (SHAPE, dict(top=-1)), (SHAPE, dict(top=65, V=100, ldl=100)), (SHAPE, dict(top=5, V=4)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=-1.0)),
    (SHAPE, dict(scale=NAN)), (SHAPE, dict(scale=INF)), (SHAPE, dict(logits=ODD)), (SHAPE, dict(dt=0, logits=FAKE + 2)),
    (SHAPE, dict(targets=FAKE + 4)), (SHAPE, dict(logp=FAKE + 2)), (SHAPE, dict(entropy=ODD)), (SHAPE, dict(rmax=ODD)), (SHAPE, dict(rlog=FAKE + 2)),
    (SHAPE, dict(top_logp=ODD)), (SHAPE, dict(top_idx=FAKE + 2)), (DTYPE, dict(dt=2)), (DTYPE, dict(idt=3)), (OK, dict(T=0)),
    (OK, dict(T=0, logits=None, targets=None, logp=None, entropy=None, rmax=None, rlog=None, top_logp=None, top_idx=None, ws=None, ws_bytes=0))])
def test_logp_forward_validation(want, kw):
    assert logp_forward(**kw) == want


def test_logp_forward_workspace():
    q = grass.logp_forward_workspace
    assert q(-1, 4, 0, 1) == q(4, 0, 0, 1) == q(4, 4, 0, 9) == q(4, 4, 5, 1) == q(4, 100, 65, 1) == q(4, 100, -1, 1) == q(BIG, 4, 0, 1) == 0
    for T, V, top, dt in ((1, 32000, 20, 1), (256, 128000, 20, 0), (3, 1000000, 64, 1), (1, 1 << 30, 0, 0)):
        need = q(T, V, top, dt)
        kw = dict(T=T, V=V, ldl=V, top=top, dt=dt)
        if not top:
            kw.update(top_logp=None, top_idx=None)
        if need:
            assert logp_forward(ws_bytes=need - 1, **kw) == logp_forward(ws=None, **kw) == logp_forward(ws=FAKE + 8, **kw) == WS


def logp_backward(**kw):
    return call(grass.lib().grass_logp_backward,
                "logits dt T V ldl targets idt scale rmax rlog dlogp entropy dentropy dlogits lddl stream".split(),
                (FAKE, 1, 8, 64, 64, FAKE, 1, 1.0, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 64, None), **kw)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(logits=None)), (NULL, dict(targets=None)), (NULL, dict(rmax=None)), (NULL, dict(rlog=None)), (NULL, dict(entropy=None)),
    (NULL, dict(dlogits=None)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=BIG)), (SHAPE, dict(V=0)), (SHAPE, dict(V=BIG)), (SHAPE, dict(ldl=63)),
    (SHAPE, dict(lddl=63)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=NAN)), (SHAPE, dict(logits=ODD)), (SHAPE, dict(dlogits=ODD)),
    (SHAPE, dict(dt=0, dlogits=FAKE + 2)), (SHAPE, dict(targets=FAKE + 4)), (SHAPE, dict(rmax=ODD)), (SHAPE, dict(rlog=FAKE + 2)),
    (SHAPE, dict(dlogp=ODD)), (SHAPE, dict(entropy=ODD)), (SHAPE, dict(dentropy=FAKE + 2)), (DTYPE, dict(dt=-1)), (DTYPE, dict(idt=2)),
    (OK, dict(T=0)), (OK, dict(T=0, targets=None, dlogp=None, entropy=None, dentropy=None, rmax=None, rlog=None, logits=None, dlogits=None))])
def test_logp_backward_validation(want, kw):
    assert logp_backward(**kw) == want


def test_binding_refuses_host_tensors():
    x, ids, f = torch.zeros(4, 4), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for bad in (lambda: grass.embed_forward(x, ids, x), lambda: grass.embed_backward(x, ids, x, None),
                lambda: grass.logp_forward(x, ids, f, None), lambda: grass.logp_backward(x, ids, f, f, f, x)):
        with pytest.raises((AssertionError, RuntimeError)):
            bad()
