"""fp64 CPU oracle of the gated linear recurrence, its gradients and the 8-bit checkpoints.

TEST INFRASTRUCTURE ONLY, like the rest of this package: the product path never imports it
and shares no code with it.

For every sequence and channel, token by token (the recurrent layer of the paper's Hawk-Mesa
hybrid), with sigma(x) = 1 / (1 + exp(-x)):

    l_t = -decay softplus(theta) sigma(r_t),  a_t = exp(l_t),  m_t = sqrt(1 - a_t^2)
    h_t = a_t h_{t-1} + m_t sigma(i_t) x_t

A reset token has a_t = 0 and m_t = 1 and reads nothing before it, whatever that holds.
"""
from __future__ import annotations

import numpy as np

from .layer_ends import _f64, sigmoid, softplus

BLOCK = 128
GROUP = 32


def _terms(x, r, i, theta, decay, reset):
    x, r, i, theta = _f64(x), _f64(r), _f64(i), _f64(theta)
    s, si = sigmoid(r), sigmoid(i)
    low = -float(decay) * softplus(theta) * s
    a, m = np.exp(low), np.sqrt(-np.expm1(2.0 * low))
    cut = np.zeros(x.shape[:2], bool) if reset is None else np.asarray(reset) != 0
    return x, theta, s, si, low, a, m, cut


def forward(x, r, i, theta, decay=8.0, reset=None, h0=None):
    """x, r, i [B, T, W]; theta [W]; reset [B, T]; h0 [B, W].  Returns a dict: y [B, T, W], h
    [B, W] (after the last token), states [B, ceil(T / BLOCK), W] (entering each block)."""
    with np.errstate(invalid="ignore", over="ignore"):
        x, theta, s, si, low, a, m, cut = _terms(x, r, i, theta, decay, reset)
        B, T, W = x.shape
        h = np.zeros((B, W)) if h0 is None else _f64(h0).copy()
        y, states = np.empty((B, T, W)), np.empty((B, -(-T // BLOCK), W))
        for t in range(T):
            if t % BLOCK == 0:
                states[:, t // BLOCK] = h
            c = cut[:, t, None]
            h = np.where(c, si[:, t] * x[:, t], a[:, t] * h + m[:, t] * si[:, t] * x[:, t])
            y[:, t] = h
    return {"y": y, "h": h, "states": states}


def backward(x, r, i, theta, states, dy, dfinal=None, decay=8.0, reset=None):
    """Gradients from dy [B, T, W] and dfinal [B, W]; the states before every token are rebuilt
    from the one that enters its block.  Returns dx, dr, di [B, T, W], dtheta [W], dh0 [B, W], and
    dtheta_size [W], the sum of the magnitudes of dtheta's terms."""
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        x, theta, s, si, low, a, m, cut = _terms(x, r, i, theta, decay, reset)
        dy, states = _f64(dy), _f64(states)
        B, T, W = x.shape
        before = np.empty((B, T, W))
        for t in range(T):
            if t % BLOCK == 0:
                h = states[:, t // BLOCK]
            before[:, t] = h
            c = cut[:, t, None]
            h = np.where(c, si[:, t] * x[:, t], a[:, t] * h + m[:, t] * si[:, t] * x[:, t])
        c = np.zeros((B, W)) if dfinal is None else _f64(dfinal).copy()
        out = {n: np.empty((B, T, W)) for n in ("dx", "dr", "di")}
        dtheta, size = np.zeros(W), np.zeros(W)
        for t in range(T - 1, -1, -1):
            hard = cut[:, t, None]
            g = dy[:, t] + c
            mt = np.where(hard, 1.0, m[:, t])
            out["dx"][:, t] = g * mt * si[:, t]
            out["di"][:, t] = g * mt * x[:, t] * si[:, t] * (1.0 - si[:, t])
            dl = np.where(hard, 0.0, g * (a[:, t] * before[:, t] - a[:, t] ** 2 / m[:, t] * si[:, t] * x[:, t]))
            out["dr"][:, t] = np.where(hard, 0.0, dl * low[:, t] * sigmoid(-_f64(r)[:, t]))
            dtheta += np.where(hard, 0.0, dl * s[:, t]).sum(axis=0)
            size += np.where(hard, 0.0, np.abs(dl * s[:, t])).sum(axis=0)
            c = np.where(hard, 0.0, a[:, t] * g)
    out["dtheta"] = -float(decay) * sigmoid(theta) * dtheta
    out["dtheta_size"] = float(decay) * sigmoid(theta) * size
    out["dh0"] = c
    return out


def checkpoint(x):
    """x [rows, width] in groups of GROUP channels: codes [rows, width] (whole numbers), exponent
    bytes [rows, groups] (E + 127, 255 for a group that is not finite), and the values that they
    stand for (fp64).  E is found by trying, from the least one up."""
    x = _f64(x)
    rows, width = x.shape
    groups = -(-width // GROUP)
    v = np.zeros((rows, groups * GROUP))
    v[:, :width] = x
    v = v.reshape(rows, groups, GROUP)
    whole = np.all(np.isfinite(v), axis=-1)
    v = np.where(whole[..., None], v, 0.0)
    amax = np.max(np.abs(v), axis=-1)
    e = np.full((rows, groups), -126)
    while True:      # the largest magnitude decides: rint keeps order
        more = (np.rint(np.ldexp(amax, -e)) > 127) & (e < 122)
        if not np.any(more):
            break
        e = np.where(more, e + 1, e)
    most = np.where(e == 122, 63, 127)[..., None]      # 64 * 2^122 is past fp32
    codes = np.clip(np.rint(np.ldexp(v, -e[..., None])), -most, most)
    value = np.where(whole[..., None], np.ldexp(codes, e[..., None]), np.nan)
    flat = (rows, groups * GROUP)
    return (codes.reshape(flat)[:, :width].astype(np.int64), np.where(whole, e + 127, 255),
            value.reshape(flat)[:, :width])
