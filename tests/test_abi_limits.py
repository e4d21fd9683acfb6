"""Sizes past one launch: the runtime counts a launch's threads along a dimension in 32 bits and past that starts
the remainder alone, without an error, so the entry points have to refuse such a call.  Each size here needs 2^32
threads or a few more and fits every other limit (and a card's memory, or nearly); nothing is launched."""
import os

import pytest

from paper_2506_05233_amd import libmesa as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return L.load()


FAR = {n: (k + 1) << 46 for k, n in enumerate(["x", "r", "i", "y", "states", "dy", "dx", "dr", "di", "ws", "th", "dth"])}


@pytest.mark.parametrize("rows,width", [(1 << 32, 1), ((1 << 32) + 256, 1), (1 << 32, 7)])
def test_checkpoint_past_one_launch(lib, rows, width):
    assert lib.mesa_checkpoint_pack(FAR["x"], rows, width, width, 1, 1 << 50, None) == L.MESA_ERR_SHAPE
    assert lib.mesa_checkpoint_unpack(1 << 50, rows, width, width, 1, FAR["x"], None) == L.MESA_ERR_SHAPE


@pytest.mark.parametrize("B,T,W", [(1 << 23, 1, 64), ((1 << 23) + 8, 1, 4), (1 << 22, 100, 65), (1 << 22, 129, 64)])
def test_recurrence_past_one_launch(lib, B, T, W):
    f = FAR
    for dtype in (0, 1):
        st = lib.mesa_recurrence_backward(f["x"], f["r"], f["i"], f["th"], 8.0, None, f["states"], f["dy"], None, B, T, W, W, dtype, dtype,
                                          W, f["dx"], f["dr"], f["di"], f["dth"], None, f["ws"], 1 << 45, None)
        assert st == L.MESA_ERR_SHAPE
        if T != 129:    # two tiles of 128 tokens, one of 256
            assert lib.mesa_recurrence(f["x"], f["r"], f["i"], f["th"], 8.0, None, None, B, T, W, W, dtype, f["y"], None, None, None, None,
                                       None, f["ws"], 1 << 45, None) == L.MESA_ERR_SHAPE


@pytest.mark.parametrize("B,W", [(1 << 24, 1024), ((1 << 22) + 1, 1025)])
def test_step_past_one_launch(lib, B, W):
    f = FAR
    assert lib.mesa_recurrence_step(f["dy"], f["x"], f["r"], f["i"], f["th"], 8.0, None, B, W, W, 1, f["states"], f["y"],
                                    None) == L.MESA_ERR_SHAPE


def test_dtheta_past_one_launch(lib):
    """Few enough workgroups of the gradient kernel, too many of the sum over its tiles."""
    f, W = FAR, 1 << 28
    assert lib.mesa_recurrence_backward(f["x"], f["r"], f["i"], f["th"], 8.0, None, f["states"], f["dy"], None, 1, 1, W, W, 0, 0, W,
                                        f["dx"], f["dr"], f["di"], f["dth"], None, f["ws"], 1 << 45, None) == L.MESA_ERR_SHAPE


def test_ends_past_one_launch(lib):
    P = [(k + 1) << 44 for k in range(30)]
    B = (1 << 32) // 256 // 3 + 1
    assert lib.mesa_frontend_backward(*P[:9], 0.99, 1e-6, B, 1, 1, 64, 64, 0, *P[9:15], 0, *P[15:24], P[24], 1 << 43,
                                      None) == L.MESA_ERR_SHAPE
    assert lib.mesa_output_norm_backward(P[0], P[1], 1e-6, P[2], 1 << 24, 1, 1, 64, 0, 0, P[3], P[4], P[5], 1 << 43,
                                         None) == L.MESA_ERR_SHAPE


# The Mesa layer's own calls: workgroups of 256 threads, several for each (sequence, head).
def test_mesa_layer_past_one_launch(lib):
    P = [(k + 1) << 46 for k in range(20)]
    big = 1 << 45
    for dtype, BH in ((0, 1 << 21), (1, 1 << 23)):      # states: a workgroup for 16 rows in fp32, two in all for bf16
        assert lib.mesa_forward(*P[:6], BH, 1, 1, 64, 64, dtype, 5, 64, P[6], P[7], big, None) == L.MESA_ERR_SHAPE
        assert lib.mesa_backward(*P[:5], BH, 1, 1, 64, 64, dtype, 5, 0, P[5], P[6], *P[7:13], P[13], big, None) == L.MESA_ERR_SHAPE
    assert lib.mesa_frontend(*P[:9], 0.99, 1e-6, 1 << 22, 8, 1, 64, 64, 0, *P[9:15], None) == L.MESA_ERR_SHAPE
    assert lib.mesa_output_norm(P[0], P[1], 1e-6, 1 << 22, 16, 1, 64, 0, P[2], None) == L.MESA_ERR_SHAPE


# With no token the states are still batch x width: their size is checked as any other's.
@pytest.mark.parametrize("B,W", [(1 << 50, 1 << 20), ((1 << 40) + 1, 1), (1 << 40, 2), (1 << 21, 1 << 20)])
def test_states_of_empty_sequences_too_large(lib, B, W):
    f = FAR
    assert lib.mesa_recurrence(None, None, None, None, 8.0, None, f["x"], B, 0, W, W, 0, None, f["y"], None, None, None, None, None, 0,
                               None) == L.MESA_ERR_SHAPE
    assert lib.mesa_recurrence_backward(None, None, None, f["th"], 8.0, None, None, None, f["dy"], B, 0, W, W, 0, 0, W, None, None, None,
                                        f["dth"], f["dx"], None, 0, None) == L.MESA_ERR_SHAPE


def test_the_status_says_so(lib):
    assert b"launch" in lib.mesa_status_string(L.MESA_ERR_SHAPE)
