"""Refusals of the recurrence's, the checkpoints' and the ends' gradients' entry points: every call
here fails validation (or has nothing to do), so nothing is launched and no GPU is needed."""
import os

import pytest

from paper_2506_05233_amd import libmesa as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return L.load()


A = {n: 0x100000000 * (k + 1) for k, n in enumerate(
    ["x", "r", "i", "theta", "reset", "h0", "y", "fh", "states", "kx", "kr", "ki", "ws", "so", "dy", "df", "dx", "dr", "di",
     "dth", "dh0", "qp", "kp", "vp", "cq", "ck", "cv", "ag", "ab", "dq", "dk", "dv", "dg", "db", "dl", "dqp", "dkp", "dvp", "dcq", "dck",
     "dcv", "dag", "dab", "o", "w"])}


def test_checkpoint_bytes():
    assert L.checkpoint_bytes(3, 100) == 304 + 16 and L.checkpoint_bytes(16, 64) == 1024 + 32
    assert L.checkpoint_bytes(0, 5) == 0 and L.checkpoint_bytes(5, -1) == 0 and L.checkpoint_bytes(1 << 40, 2) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.MESA_ERR_SHAPE), (dict(width=-1), L.MESA_ERR_SHAPE), (dict(stride=63), L.MESA_ERR_SHAPE),
    (dict(rows=1 << 40), L.MESA_ERR_SHAPE), (dict(dtype=2), L.MESA_ERR_UNSUPPORTED), (dict(dtype=-1), L.MESA_ERR_UNSUPPORTED),
    (dict(x=None), L.MESA_ERR_NULL), (dict(ck=None), L.MESA_ERR_NULL), (dict(ck=A["kx"] + 8), L.MESA_ERR_ARG),
    (dict(x=A["x"] + 2), L.MESA_ERR_ARG), (dict(ck=A["x"]), L.MESA_ERR_ARG), (dict(ck=A["x"] + 10 * 256 - 16), L.MESA_ERR_ARG),
    (dict(rows=0, x=None, ck=None), L.MESA_OK), (dict(width=0, x=None, ck=None), L.MESA_OK)])
def test_checkpoint_refuses(lib, kw, status):
    a = dict(x=A["x"], rows=10, width=64, stride=64, dtype=0, ck=A["kx"])
    a.update(kw)
    assert lib.mesa_checkpoint_pack(a["x"], a["rows"], a["width"], a["stride"], a["dtype"], a["ck"], None) == status
    assert lib.mesa_checkpoint_unpack(a["ck"], a["rows"], a["width"], a["stride"], a["dtype"], a["x"], None) == status


def _rec(lib, **kw):
    a = dict(x=A["x"], r=A["r"], i=A["i"], theta=A["theta"], decay=8.0, reset=None, h0=None, B=2, T=600, W=64, stride=64, dtype=0,
             y=A["y"], fh=None, states=None, kx=None, kr=None, ki=None, ws=A["ws"], wsb=1 << 40)
    a.update(kw)
    return lib.mesa_recurrence(a["x"], a["r"], a["i"], a["theta"], a["decay"], a["reset"], a["h0"], a["B"], a["T"], a["W"],
                               a["stride"], a["dtype"], a["y"], a["fh"], a["states"], a["kx"], a["kr"], a["ki"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), L.MESA_ERR_SHAPE), (dict(T=-1), L.MESA_ERR_SHAPE), (dict(W=-1), L.MESA_ERR_SHAPE),
    (dict(stride=63), L.MESA_ERR_SHAPE), (dict(T=1 << 62), L.MESA_ERR_SHAPE), (dict(B=1 << 31, T=128), L.MESA_ERR_SHAPE),
    (dict(stride=1 << 39), L.MESA_ERR_SHAPE),
    (dict(dtype=2), L.MESA_ERR_UNSUPPORTED), (dict(decay=0.0), L.MESA_ERR_ARG), (dict(decay=-1.0), L.MESA_ERR_ARG),
    (dict(decay=float("nan")), L.MESA_ERR_ARG), (dict(decay=float("inf")), L.MESA_ERR_ARG),
    (dict(x=None), L.MESA_ERR_NULL), (dict(i=None), L.MESA_ERR_NULL), (dict(theta=None), L.MESA_ERR_NULL),
    (dict(y=None), L.MESA_ERR_NULL), (dict(kx=A["kx"]), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL),
    (dict(wsb=8), L.MESA_ERR_WORKSPACE), (dict(x=A["x"] + 2), L.MESA_ERR_ARG), (dict(h0=A["h0"] + 2), L.MESA_ERR_ARG),
    (dict(kx=A["kx"] + 4, kr=A["kr"], ki=A["ki"]), L.MESA_ERR_ARG), (dict(ws=A["ws"] + 8), L.MESA_ERR_ARG),
    (dict(y=A["x"]), L.MESA_ERR_ARG), (dict(fh=A["theta"]), L.MESA_ERR_ARG), (dict(states=A["y"] + 1024), L.MESA_ERR_ARG),
    (dict(h0=A["h0"], fh=A["h0"]), L.MESA_ERR_ARG), (dict(ws=A["y"]), L.MESA_ERR_ARG),
    (dict(stride=256, y=A["x"] + 256), L.MESA_ERR_ARG),        # a dense output between the rows of a spaced input
    (dict(B=0, x=None, y=None), L.MESA_OK), (dict(W=0, x=None, y=None, theta=None), L.MESA_OK)])
def test_recurrence_refuses(lib, kw, status):
    assert _rec(lib, **kw) == status


def test_recurrence_workspace():
    assert L.recurrence_workspace_bytes(2, 1, 64) == 0 and L.recurrence_workspace_bytes(0, 9999, 64) == 0
    assert L.recurrence_workspace_bytes(2, 5000, 64) > 0 and L.recurrence_workspace_bytes(-1, 5, 5) == 0
    assert L.recurrence_backward_workspace_bytes(2, 1, 64) >= 2 * 64 * 4


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), L.MESA_ERR_SHAPE), (dict(stride=7), L.MESA_ERR_SHAPE), (dict(dtype=2), L.MESA_ERR_UNSUPPORTED),
    (dict(decay=0.0), L.MESA_ERR_ARG), (dict(state=None), L.MESA_ERR_NULL), (dict(so=None), L.MESA_ERR_NULL),
    (dict(r=None), L.MESA_ERR_NULL), (dict(state=A["h0"] + 2), L.MESA_ERR_ARG), (dict(so=A["h0"] + 4), L.MESA_ERR_ARG),
    (dict(y=A["h0"]), L.MESA_ERR_ARG), (dict(y=A["x"]), L.MESA_ERR_ARG), (dict(so=A["theta"]), L.MESA_ERR_ARG),
    (dict(B=0, state=None), L.MESA_OK)])
def test_step_refuses(lib, kw, status):
    a = dict(state=A["h0"], x=A["x"], r=A["r"], i=A["i"], theta=A["theta"], decay=8.0, B=3, W=8, stride=8, dtype=0, so=A["so"], y=A["y"])
    a.update(kw)
    assert lib.mesa_recurrence_step(a["state"], a["x"], a["r"], a["i"], a["theta"], a["decay"], None, a["B"], a["W"], a["stride"],
                                    a["dtype"], a["so"], a["y"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), L.MESA_ERR_SHAPE), (dict(stride=63), L.MESA_ERR_SHAPE), (dict(gs=63), L.MESA_ERR_SHAPE),
    (dict(dtype=3), L.MESA_ERR_UNSUPPORTED), (dict(gdtype=2), L.MESA_ERR_UNSUPPORTED), (dict(decay=0.0), L.MESA_ERR_ARG),
    (dict(states=None), L.MESA_ERR_NULL), (dict(dy=None), L.MESA_ERR_NULL), (dict(dth=None), L.MESA_ERR_NULL),
    (dict(ws=None), L.MESA_ERR_NULL), (dict(wsb=16), L.MESA_ERR_WORKSPACE), (dict(dtype=2, x=A["x"] + 4), L.MESA_ERR_ARG),
    (dict(dy=A["dy"] + 2), L.MESA_ERR_ARG), (dict(dx=A["x"]), L.MESA_ERR_ARG), (dict(dr=A["dx"]), L.MESA_ERR_ARG),
    (dict(gs=128, dr=A["dx"] + 128), L.MESA_ERR_ARG),          # slices that overlap: 64 channels are 256 bytes
    (dict(dh0=A["df"], df=A["df"]), L.MESA_ERR_ARG), (dict(ws=A["dx"]), L.MESA_ERR_ARG)])
def test_recurrence_backward_refuses(lib, kw, status):
    a = dict(x=A["x"], r=A["r"], i=A["i"], theta=A["theta"], decay=8.0, reset=None, states=A["states"], dy=A["dy"], df=None, B=2,
             T=300, W=64, stride=64, dtype=0, gdtype=0, gs=64, dx=A["dx"], dr=A["dr"], di=A["di"], dth=A["dth"], dh0=None,
             ws=A["ws"], wsb=1 << 40)
    a.update(kw)
    assert lib.mesa_recurrence_backward(a["x"], a["r"], a["i"], a["theta"], a["decay"], a["reset"], a["states"], a["dy"], a["df"],
                                        a["B"], a["T"], a["W"], a["stride"], a["dtype"], a["gdtype"], a["gs"], a["dx"], a["dr"],
                                        a["di"], a["dth"], a["dh0"], a["ws"], a["wsb"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), L.MESA_ERR_SHAPE), (dict(dk=96), L.MESA_ERR_UNSUPPORTED), (dict(dtype=3), L.MESA_ERR_UNSUPPORTED),
    (dict(gdtype=2), L.MESA_ERR_UNSUPPORTED), (dict(cap=1.5), L.MESA_ERR_ARG), (dict(eps=-1.0), L.MESA_ERR_ARG),
    (dict(B=1 << 20, T=1 << 20), L.MESA_ERR_SHAPE), (dict(qp=None), L.MESA_ERR_NULL), (dict(vp=None), L.MESA_ERR_NULL),
    (dict(dcv=None), L.MESA_ERR_NULL), (dict(dl=None), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL),
    (dict(wsb=16), L.MESA_ERR_WORKSPACE), (dict(qp=A["qp"] + 8), L.MESA_ERR_ARG), (dict(ag=A["ag"] + 2), L.MESA_ERR_ARG),
    (dict(dqp=A["dq"]), L.MESA_ERR_ARG), (dict(dkp=A["dqp"]), L.MESA_ERR_ARG), (dict(dcq=A["cq"]), L.MESA_ERR_ARG),
    (dict(H=0, qp=None, dth=None), L.MESA_OK)])
def test_frontend_backward_refuses(lib, kw, status):
    a = dict(qp=A["qp"], kp=A["kp"], vp=A["vp"], cv=A["cv"], ag=A["ag"], cap=0.99, eps=1e-6, B=2, H=3, T=50, dk=64, dtype=0, gdtype=0,
             dl=A["dl"], dqp=A["dqp"], dkp=A["dkp"], dcq=A["dcq"], dcv=A["dcv"], dth=A["dth"], ws=A["ws"], wsb=1 << 40)
    a.update(kw)
    assert lib.mesa_frontend_backward(a["qp"], a["kp"], a["vp"], A["cq"], A["ck"], a["cv"], a["ag"], A["ab"], A["theta"], a["cap"],
                                      a["eps"], a["B"], a["H"], a["T"], a["dk"], 128, a["dtype"], A["dq"], A["dk"], A["dv"], A["dg"],
                                      A["db"], a["dl"], a["gdtype"], a["dqp"], a["dkp"], A["dvp"], a["dcq"], A["dck"], a["dcv"],
                                      A["dag"], A["dab"], a["dth"], a["ws"], a["wsb"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), L.MESA_ERR_SHAPE), (dict(dv=32), L.MESA_ERR_UNSUPPORTED), (dict(dtype=1), L.MESA_ERR_UNSUPPORTED),
    (dict(gdtype=2), L.MESA_ERR_UNSUPPORTED), (dict(eps=float("inf")), L.MESA_ERR_ARG), (dict(o=None), L.MESA_ERR_NULL),
    (dict(w=None), L.MESA_ERR_NULL), (dict(ws=None), L.MESA_ERR_NULL), (dict(wsb=8), L.MESA_ERR_WORKSPACE),
    (dict(o=A["o"] + 4), L.MESA_ERR_ARG), (dict(do=A["o"]), L.MESA_ERR_ARG), (dict(do=A["ws"]), L.MESA_ERR_ARG),
    (dict(H=0, o=None, w=None), L.MESA_OK)])
def test_output_norm_backward_refuses(lib, kw, status):
    a = dict(o=A["o"], w=A["w"], eps=1e-6, B=2, H=3, T=50, dv=64, dtype=0, gdtype=0, do=A["dx"], ws=A["ws"], wsb=1 << 40)
    a.update(kw)
    assert lib.mesa_output_norm_backward(a["o"], a["w"], a["eps"], A["dy"], a["B"], a["H"], a["T"], a["dv"], a["dtype"], a["gdtype"],
                                         a["do"], A["dth"], a["ws"], a["wsb"], None) == status
