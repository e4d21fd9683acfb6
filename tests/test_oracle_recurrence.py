"""Pins of the recurrence's, the checkpoints' and the ends' gradients' fp64 oracle (CPU): worked
values, identities that do not use its formulas, and central differences."""
import numpy as np
import pytest

from oracle import layer_ends as E
from oracle import recurrence as R


def _inputs(B, T, W, seed, resets=False):
    rng = np.random.default_rng(seed)
    x, r, i = (rng.standard_normal((B, T, W)) for _ in range(3))
    reset = (rng.random((B, T)) < 0.2).astype(np.uint8) if resets else None
    return x, r, i, rng.standard_normal(W) - 1.0, reset, rng.standard_normal((B, W)), rng


def test_worked_recurrence():
    """theta = 0, decay = 2, r = 0: a = exp(-2 ln 2 / 2) = 1/2, m = sqrt(3)/2; i = 0 halves x."""
    x = np.array([[[8.0], [0.0], [4.0]]])
    z = np.zeros_like(x)
    f = R.forward(x, z, z, np.zeros(1), decay=2.0, h0=np.array([[2.0]]))
    m = np.sqrt(0.75)
    want = [1.0 + 4.0 * m, 0.5 + 2.0 * m, 0.25 + 1.0 * m + 2.0 * m]
    assert np.allclose(f["y"][0, :, 0], want, rtol=1e-15) and np.allclose(f["h"], want[-1], rtol=1e-15)
    f = R.forward(x, z, z, np.zeros(1), decay=2.0, h0=np.array([[np.nan]]), reset=np.array([[1, 0, 1]]))
    assert np.allclose(f["y"][0, :, 0], [4.0, 2.0, 2.0], rtol=1e-15)


def test_recurrence_equals_the_unrolled_sum():
    x, r, i, theta, _, h0, _ = _inputs(2, 40, 5, 1)
    low = -8.0 * np.log1p(np.exp(theta)) / (1.0 + np.exp(-r))
    b = np.sqrt(1.0 - np.exp(2.0 * low)) / (1.0 + np.exp(-i)) * x
    total = np.cumsum(low, axis=1)
    want = np.exp(total) * h0[:, None]
    for t in range(40):
        want[:, t] += np.sum(np.exp(total[:, t:t + 1] - total[:, :t + 1]) * b[:, :t + 1], axis=1)
    assert np.allclose(R.forward(x, r, i, theta, h0=h0)["y"], want, rtol=1e-11, atol=1e-13)


def test_reset_separates_documents_and_states_enter_blocks():
    x, r, i, theta, _, h0, _ = _inputs(1, 300, 3, 2)
    reset = np.zeros((1, 300), np.uint8)
    reset[0, 130] = 1
    f = R.forward(x, r, i, theta, reset=reset, h0=h0)
    first = R.forward(x[:, :130], r[:, :130], i[:, :130], theta, h0=h0)
    assert np.array_equal(f["y"][:, :130], first["y"])
    r2 = r.copy()
    r2[0, 130] = -1e4       # a and m of that token: a document's own start, scaled by 1 / m
    one = E.sigmoid(i[:, 130]) * x[:, 130]
    rest = R.forward(x[:, 131:], r[:, 131:], i[:, 131:], theta, h0=one)
    assert np.allclose(f["y"][:, 130], one) and np.allclose(f["y"][:, 131:], rest["y"], rtol=1e-13)
    assert np.array_equal(f["states"][:, 0], h0) and np.array_equal(f["states"][:, 1], f["y"][:, 127])
    assert np.array_equal(f["states"][:, 2], f["y"][:, 255]) and f["states"].shape[1] == 3


@pytest.mark.parametrize("T,resets", [(1, False), (9, True), (135, False), (135, True)])
def test_recurrence_gradients_against_differences(T, resets):
    x, r, i, theta, reset, h0, rng = _inputs(2, T, 3, 3 + T, resets)
    dy, dfin = rng.standard_normal(x.shape), rng.standard_normal(h0.shape)

    def loss(x, r, i, theta, h0):
        f = R.forward(x, r, i, theta, reset=reset, h0=h0)
        return np.sum(f["y"] * dy) + np.sum(f["h"] * dfin)

    args = {"dx": x, "dr": r, "di": i, "dtheta": theta, "dh0": h0}
    got = R.backward(x, r, i, theta, R.forward(x, r, i, theta, reset=reset, h0=h0)["states"], dy, dfin, reset=reset)
    for k, name in enumerate(args):
        a = args[name]
        for e in rng.choice(a.size, size=min(a.size, 25), replace=False):
            step = np.zeros(a.size)
            step[e] = 1e-6
            step = step.reshape(a.shape)
            hi, lo = [v + step if q == k else v for q, v in enumerate(args.values())], [v - step if q == k else v for q, v in enumerate(args.values())]
            want = (loss(*hi) - loss(*lo)) / 2e-6
            assert abs(got[name].reshape(-1)[e] - want) <= 1e-7 * max(1.0, abs(want)), (name, e)


def test_checkpoint_by_hand():
    x = np.zeros((1, 70))
    x[0, :32] = np.arange(32) * 4.0 + 3.5          # largest 127.5: one more power of two
    x[0, 32:64] = np.linspace(-127.0, 127.0, 32)
    x[0, 64:] = [0.5, 1.5, 2.5, -0.5, -1.5, 127.0]  # halves go to even
    codes, byte, value = R.checkpoint(x)
    assert list(byte[0]) == [128, 127, 127]
    assert list(codes[0, 64:]) == [0, 2, 2, 0, -2, 127]
    assert codes[0, 31] == 64 and value[0, 31] == 128.0 and np.max(np.abs(value[0, :32] - x[0, :32])) <= 1.0
    x[0, 40] = np.inf
    codes, byte, value = R.checkpoint(x)
    assert list(byte[0]) == [128, 255, 127] and np.all(np.isnan(value[0, 32:64])) and np.all(np.isfinite(value[0, 64:]))
    top = np.array([[np.finfo(np.float32).max, 2.0 ** 121]])
    codes, byte, value = R.checkpoint(top)
    assert byte[0, 0] == 249 and list(codes[0]) == [63, 0] and value[0, 0] == 63 * 2.0 ** 122
    codes, byte, value = R.checkpoint(np.array([[0.0, -0.0], [2.0 ** -149, 2.0 ** -120]]))
    assert list(byte[:, 0]) == [1, 1] and list(codes[1]) == [0, 64] and not np.any(value[0])


def test_checkpoint_error_is_half_a_step():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((50, 96)) * np.exp(rng.normal(0, 10, (50, 96)))
    codes, byte, value = R.checkpoint(x)
    scale = np.repeat(2.0 ** (byte - 127.0), 32, axis=1)
    amax = np.repeat(np.abs(x).reshape(50, 3, 32).max(-1), 32, axis=1)
    assert np.all(np.abs(value - x) <= scale / 2) and np.all(scale <= amax / 63.5) and np.max(np.abs(codes)) <= 127


@pytest.mark.parametrize("T,conv_v", [(1, True), (3, False), (9, True)])
def test_frontend_gradients_against_differences(T, conv_v):
    rng = np.random.default_rng(T)
    B, H, dk, dv = 2, 2, 4, 3
    names = ["qp", "kp", "vp", "conv_q", "conv_k", "conv_v", "a_gamma", "a_beta", "theta"]
    args = [rng.standard_normal(s) for s in ((B, T, H, dk), (B, T, H, dk), (B, T, H, dv), (H * dk, 4), (H * dk, 4), (H * dv, 4),
                                             (B, T, H), (B, T, H), (H, dk))]
    if not conv_v:
        args[5] = None
    outs = ["q", "k", "v", "gamma", "beta", "lam"]
    f = E.frontend(*args, gamma_cap=0.6)
    d = [rng.standard_normal(f[n].shape) for n in outs]
    got = E.frontend_backward(*args, *d, gamma_cap=0.6)

    def loss(a):
        f = E.frontend(*a, gamma_cap=0.6)
        return sum(np.sum(f[n] * g) for n, g in zip(outs, d))

    for k, n in enumerate(names):
        if args[k] is None:
            assert got["d" + n] is None
            continue
        for e in rng.choice(args[k].size, size=min(args[k].size, 20), replace=False):
            step = np.zeros(args[k].size)
            step[e] = 1e-6
            step = step.reshape(args[k].shape)
            want = (loss([a + step if q == k else a for q, a in enumerate(args)]) -
                    loss([a - step if q == k else a for q, a in enumerate(args)])) / 2e-6
            assert abs(got["d" + n].reshape(-1)[e] - want) <= 2e-7 * max(1.0, abs(want)), (n, e)


def test_output_norm_gradients_against_differences():
    rng = np.random.default_rng(8)
    o, w, dy = rng.standard_normal((2, 3, 4, 5)), rng.standard_normal((3, 5)), rng.standard_normal((2, 4, 3, 5))
    do, dw = E.output_norm_backward(o, w, dy, 1e-3)
    for a, g, which in ((o, do, 0), (w, dw, 1)):
        for e in rng.choice(a.size, size=15, replace=False):
            step = np.zeros(a.size)
            step[e] = 1e-6
            step = step.reshape(a.shape)
            hi = E.output_norm(o + step, w, 1e-3) if which == 0 else E.output_norm(o, w + step, 1e-3)
            lo = E.output_norm(o - step, w, 1e-3) if which == 0 else E.output_norm(o, w - step, 1e-3)
            want = np.sum((hi - lo) * dy) / 2e-6
            assert abs(g.reshape(-1)[e] - want) <= 1e-7 * max(1.0, abs(want))
