"""Refusals of the embedding's and the cross entropy's entry points: every call here fails validation (or has nothing to
do), so nothing is launched and no GPU is needed."""
import os

import pytest

from paper_2506_05233_amd import libmesa as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return L.load()


A = {n: 0x100000000 * (k + 1) for k, n in enumerate(["e", "t", "y", "dy", "de", "ws", "h", "loss", "lse", "best", "up", "dh"])}
NAN, INF = float("nan"), float("inf")


def _embed(lib, **kw):
    a = dict(e=A["e"], t=A["t"], tb=8, scale=1.0, rows=10, V=50, W=64, es=64, dt=0, od=0, os=64, y=A["y"])
    a.update(kw)
    return lib.mesa_embedding(a["e"], a["t"], a["tb"], a["scale"], a["rows"], a["V"], a["W"], a["es"], a["dt"], a["od"], a["os"], a["y"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.MESA_ERR_SHAPE), (dict(V=-1), L.MESA_ERR_SHAPE), (dict(W=-1), L.MESA_ERR_SHAPE), (dict(es=63), L.MESA_ERR_SHAPE),
    (dict(os=63), L.MESA_ERR_SHAPE), (dict(rows=(1 << 24) + 1), L.MESA_ERR_SHAPE), (dict(V=(1 << 31) - 1), L.MESA_ERR_SHAPE),
    (dict(W=(1 << 16) + 1, es=1 << 17, os=1 << 17), L.MESA_ERR_SHAPE), (dict(es=1 << 36), L.MESA_ERR_SHAPE),
    (dict(dt=2), L.MESA_ERR_UNSUPPORTED), (dict(od=2), L.MESA_ERR_UNSUPPORTED), (dict(tb=2), L.MESA_ERR_UNSUPPORTED),
    (dict(scale=NAN), L.MESA_ERR_ARG), (dict(scale=INF), L.MESA_ERR_ARG), (dict(e=None), L.MESA_ERR_NULL),
    (dict(t=None), L.MESA_ERR_NULL), (dict(y=None), L.MESA_ERR_NULL), (dict(e=A["e"] + 2), L.MESA_ERR_ARG),
    (dict(y=A["y"] + 2), L.MESA_ERR_ARG), (dict(t=A["t"] + 4), L.MESA_ERR_ARG), (dict(y=A["e"] + 256), L.MESA_ERR_ARG),
    (dict(y=A["t"]), L.MESA_ERR_ARG), (dict(rows=0, t=None, y=None), L.MESA_OK), (dict(W=0, y=None), L.MESA_OK)])
def test_embedding_refuses(lib, kw, status):
    assert _embed(lib, **kw) == status


def _embed_grad(lib, **kw):
    a = dict(t=A["t"], tb=4, dy=A["dy"], scale=1.0, rows=100, V=50, W=64, ds=64, gd=1, td=1, es=64, acc=0, de=A["de"], ws=A["ws"], wsb=1 << 30)
    a.update(kw)
    return lib.mesa_embedding_backward(a["t"], a["tb"], a["dy"], a["scale"], a["rows"], a["V"], a["W"], a["ds"], a["gd"], a["td"], a["es"],
                                       a["acc"], a["de"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.MESA_ERR_SHAPE), (dict(ds=63), L.MESA_ERR_SHAPE), (dict(es=63), L.MESA_ERR_SHAPE), (dict(gd=2), L.MESA_ERR_UNSUPPORTED),
    (dict(td=3), L.MESA_ERR_UNSUPPORTED), (dict(tb=1), L.MESA_ERR_UNSUPPORTED), (dict(scale=NAN), L.MESA_ERR_ARG), (dict(t=None), L.MESA_ERR_NULL),
    (dict(dy=None), L.MESA_ERR_NULL), (dict(de=None), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL), (dict(wsb=64), L.MESA_ERR_WORKSPACE),
    (dict(ws=A["ws"] + 8), L.MESA_ERR_ARG), (dict(dy=A["dy"] + 1), L.MESA_ERR_ARG), (dict(de=A["de"] + 1), L.MESA_ERR_ARG),
    (dict(t=A["t"] + 2), L.MESA_ERR_ARG), (dict(de=A["dy"] + 128), L.MESA_ERR_ARG), (dict(ws=A["de"]), L.MESA_ERR_ARG),
    (dict(ws=A["t"] + 16), L.MESA_ERR_ARG), (dict(V=0, de=None), L.MESA_OK), (dict(W=0, de=None), L.MESA_OK),
    (dict(rows=0, acc=1, t=None, dy=None, de=None), L.MESA_OK)])
def test_embedding_backward_refuses(lib, kw, status):
    assert _embed_grad(lib, **kw) == status


def _loss(lib, **kw):
    a = dict(h=A["h"], e=A["e"], t=A["t"], tb=8, cap=30.0, rows=100, V=50, W=64, hs=64, es=64, dt=1, loss=A["loss"], lse=A["lse"], best=None,
             ws=A["ws"], wsb=1 << 30)
    a.update(kw)
    return lib.mesa_cross_entropy(a["h"], a["e"], a["t"], a["tb"], a["cap"], a["rows"], a["V"], a["W"], a["hs"], a["es"], a["dt"], a["loss"],
                                  a["lse"], a["best"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.MESA_ERR_SHAPE), (dict(V=0), L.MESA_ERR_SHAPE), (dict(W=0), L.MESA_ERR_SHAPE), (dict(hs=63), L.MESA_ERR_SHAPE),
    (dict(es=63), L.MESA_ERR_SHAPE), (dict(dt=2), L.MESA_ERR_UNSUPPORTED), (dict(tb=3), L.MESA_ERR_UNSUPPORTED), (dict(cap=-1.0), L.MESA_ERR_ARG),
    (dict(cap=NAN), L.MESA_ERR_ARG), (dict(cap=INF), L.MESA_ERR_ARG), (dict(cap=1e-40), L.MESA_ERR_ARG), (dict(h=None), L.MESA_ERR_NULL), (dict(e=None), L.MESA_ERR_NULL),
    (dict(lse=None), L.MESA_ERR_NULL), (dict(loss=None), L.MESA_ERR_NULL), (dict(t=None), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL),
    (dict(wsb=64), L.MESA_ERR_WORKSPACE), (dict(h=A["h"] + 1), L.MESA_ERR_ARG), (dict(lse=A["lse"] + 2), L.MESA_ERR_ARG),
    (dict(best=A["best"] + 2), L.MESA_ERR_ARG), (dict(t=A["t"] + 4), L.MESA_ERR_ARG), (dict(ws=A["ws"] + 4), L.MESA_ERR_ARG),
    (dict(lse=A["loss"]), L.MESA_ERR_ARG), (dict(best=A["lse"] + 4), L.MESA_ERR_ARG), (dict(loss=A["h"] + 16), L.MESA_ERR_ARG),
    (dict(ws=A["e"] + 16), L.MESA_ERR_ARG), (dict(rows=0, h=None, lse=None), L.MESA_OK)])
def test_cross_entropy_refuses(lib, kw, status):
    assert _loss(lib, **kw) == status


def _loss_grad(lib, **kw):
    a = dict(h=A["h"], e=A["e"], t=A["t"], tb=8, lse=A["lse"], up=A["up"], cap=30.0, rows=100, V=50, W=64, hs=64, es=64, dt=0, dhs=64, des=64,
             dh=A["dh"], de=A["de"], ws=A["ws"], wsb=1 << 30)
    a.update(kw)
    return lib.mesa_cross_entropy_backward(a["h"], a["e"], a["t"], a["tb"], a["lse"], a["up"], a["cap"], a["rows"], a["V"], a["W"], a["hs"],
                                           a["es"], a["dt"], a["dhs"], a["des"], a["dh"], a["de"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.MESA_ERR_SHAPE), (dict(V=0), L.MESA_ERR_SHAPE), (dict(W=0), L.MESA_ERR_SHAPE), (dict(hs=63), L.MESA_ERR_SHAPE),
    (dict(es=63), L.MESA_ERR_SHAPE), (dict(dhs=63), L.MESA_ERR_SHAPE), (dict(des=63), L.MESA_ERR_SHAPE), (dict(dt=2), L.MESA_ERR_UNSUPPORTED),
    (dict(tb=0), L.MESA_ERR_UNSUPPORTED), (dict(cap=-1.0), L.MESA_ERR_ARG), (dict(cap=INF), L.MESA_ERR_ARG), (dict(cap=1e-40), L.MESA_ERR_ARG), (dict(h=None), L.MESA_ERR_NULL),
    (dict(t=None), L.MESA_ERR_NULL), (dict(lse=None), L.MESA_ERR_NULL), (dict(up=None), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL),
    (dict(wsb=64), L.MESA_ERR_WORKSPACE), (dict(dh=A["dh"] + 2), L.MESA_ERR_ARG), (dict(de=A["de"] + 2), L.MESA_ERR_ARG),
    (dict(up=A["up"] + 2), L.MESA_ERR_ARG), (dict(ws=A["ws"] + 4), L.MESA_ERR_ARG), (dict(dh=A["h"]), L.MESA_ERR_ARG),
    (dict(de=A["e"]), L.MESA_ERR_ARG), (dict(de=A["dh"] + 256), L.MESA_ERR_ARG), (dict(ws=A["dh"]), L.MESA_ERR_ARG),
    (dict(dh=None, de=None), L.MESA_OK), (dict(rows=0, V=0), L.MESA_OK), (dict(rows=0, dh=None, de=None, h=None), L.MESA_OK)])
def test_cross_entropy_backward_refuses(lib, kw, status):
    assert _loss_grad(lib, **kw) == status


def test_workspace_bytes():
    assert L.embedding_backward_workspace_bytes(-1, 5, 5) == 0 and L.embedding_backward_workspace_bytes(10, 0, 5) == 0
    assert L.embedding_backward_workspace_bytes(0, 100, 64) == 0 and L.embedding_backward_workspace_bytes(1000, 5, 64) >= 16000
    for f in (L.cross_entropy_workspace_bytes, L.cross_entropy_backward_workspace_bytes):
        assert f(0, 5, 5, 0) == 0 and f(5, 0, 5, 0) == 0 and f(5, 5, 5, 2) == 0 and f(1 << 25, 5, 5, 0) == 0
        assert 0 < f(1, 1, 1, 1) < 1 << 20
    # dz is held a piece at a time, the logits never: 16384 rows of 50257 would be 3.3 GB of them
    assert L.cross_entropy_backward_workspace_bytes(16384, 50257, 2048, 1) < 700 << 20
    assert L.cross_entropy_workspace_bytes(16384, 50257, 2048, 1) < 400 << 20


def test_binding_checks():
    torch = pytest.importorskip("torch")
    e, t = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: L.embedding(e, t), lambda: L.embedding_backward(t, e, 5), lambda: L.cross_entropy(e, e, t),
                 lambda: L.cross_entropy_backward(e, e, t, e, e)):
        with pytest.raises(ValueError):     # host tensors
            call()
    with pytest.raises(TypeError):
        L.embedding([1.0], t)
