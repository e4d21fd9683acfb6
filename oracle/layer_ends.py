"""fp64 CPU oracle of the Mesa layer's front and back end (MesaNet, arXiv 2506.05233).

TEST INFRASTRUCTURE ONLY.  Only ``tests/``, ``__graft_entry__.smoke()`` and the
CPU-baseline leg of ``bench.py`` may import this module; the product path never
imports, links or calls it, and it shares no code with that path.

What it computes, written from App. E ("A Full Description of the Mesa Layer")
and App. G.5 ("Notes on precision used in the CG-solver"), per head h:

  front end, from the projections q_t = W_q e_t, k_t = W_k e_t, v_t = W_v e_t and
  the gate projections a_t^gamma = e_t W_gamma + b_gamma, a_t^beta = e_t W_beta + b_beta:
    short convolution in time, window 4:  x_t <- sum_{i=0..3} w_{i+1} x_{t-i}
        (one filter per feature channel; x_s = 0 before the first token)
    SiLU(x) = x sigma(x), then keys and queries (not values) normalised to unit L2 norm
    input gate beta_t = sigma(a_t^beta)
    forget gate gamma_t = sigma(a_t^gamma) s_t,  s_t = 1 - (1 - b_gamma) beta_t^2
        (the cap of App. G.5: with beta_t = 1 the gate stays below b_gamma = 0.9975)
    regulariser Lambda = 0.25 + softplus(theta)   (App. G.5's lower bound 0.25)
  back end: the head's output through its RMSNorm before the output projection,
    y_t = o_t / sqrt(mean(o_t^2) + eps) * w_h.

Readings where the paper is silent:
  - the convolution is depthwise (one 4-tap filter per channel of every head) and
    causal with zeros before the sequence start; the paper's w_{i+1} multiplies x_{t-i};
  - the values take the convolution and SiLU only when a filter for them is given
    (App. E convolves "them" after all three projections, App. G.2 convolves keys and
    queries), and are never normalised;
  - the L2 normalisation divides by sqrt(|x|^2 + eps_l2) (eps_l2 small, so a zero
    vector stays zero); the RMSNorm divides by sqrt(mean(o^2) + eps_rms) and scales by
    a learnable weight per head and feature;
  - the input gate enters the cap as beta_t^2 exactly as printed.

Layouts: projections [B, T, H, d] (the heads of a token side by side, as a projection
produces them); the layer's inputs q, k [B, H, T, d_k], v [B, H, T, d_v], gamma, beta
[B, H, T], Lambda [H, d_k]; the back end's output [B, T, H, d_v].
"""
from __future__ import annotations

import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def sigmoid(x):
    """sigma(x) = 1 / (1 + exp(-x))."""
    return 1.0 / (1.0 + np.exp(-_f64(x)))


def silu(x):
    """SiLU(x) = x sigma(x) (App. E)."""
    x = _f64(x)
    return x * sigmoid(x)


def softplus(x):
    """log(1 + exp(x)), evaluated as max(x, 0) + log(1 + exp(-|x|))."""
    x = _f64(x)
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def short_conv(x, w):
    """Causal convolution of window 4 along time (App. E): y_t = sum_{i=0..3} w[c, i] x_{t-i}
    for every channel c, with x_s = 0 for s < 0.  x [..., T, C], w [C, 4]."""
    x, w = _f64(x), _f64(w)
    T = x.shape[-2]
    y = np.zeros_like(x)
    for i in range(4):
        if i < T:
            y[..., i:, :] += w[:, i] * x[..., :T - i, :]
    return y


def l2_normalize(x, eps):
    """x / sqrt(|x|^2 + eps) over the last axis."""
    x = _f64(x)
    return x / np.sqrt(np.sum(x * x, axis=-1, keepdims=True) + eps)


def gates(a_gamma, a_beta, gamma_cap):
    """Input and forget gates of App. E with the cap of App. G.5:
    beta = sigma(a_beta), gamma = sigma(a_gamma) (1 - (1 - gamma_cap) beta^2)."""
    beta = sigmoid(a_beta)
    gamma = sigmoid(a_gamma) * (1.0 - (1.0 - float(gamma_cap)) * beta * beta)
    return gamma, beta


def regulariser(theta):
    """Lambda = 0.25 + softplus(theta) (App. G.5)."""
    return 0.25 + softplus(theta)


def frontend(qp, kp, vp, conv_q, conv_k, conv_v, a_gamma, a_beta, theta, gamma_cap=0.9975,
             l2_eps=1e-6):
    """The layer's inputs from the projections.

    qp, kp [B, T, H, d_k], vp [B, T, H, d_v]; conv_q, conv_k [H*d_k, 4], conv_v
    [H*d_v, 4] or None; a_gamma, a_beta [B, T, H]; theta [H, d_k].
    Returns a dict: q, k [B, H, T, d_k], v [B, H, T, d_v], gamma, beta [B, H, T],
    lam [H, d_k].
    """
    qp, kp, vp = _f64(qp), _f64(kp), _f64(vp)
    B, T, H, dk = qp.shape
    dv = vp.shape[-1]

    def conv_silu(x, w, d):
        y = short_conv(x.reshape(B, T, H * d), w)
        return silu(y).reshape(B, T, H, d)

    q = l2_normalize(conv_silu(qp, conv_q, dk), l2_eps)
    k = l2_normalize(conv_silu(kp, conv_k, dk), l2_eps)
    v = conv_silu(vp, conv_v, dv) if conv_v is not None else vp
    gamma, beta = gates(a_gamma, a_beta, gamma_cap)
    return {
        "q": np.ascontiguousarray(q.transpose(0, 2, 1, 3)),
        "k": np.ascontiguousarray(k.transpose(0, 2, 1, 3)),
        "v": np.ascontiguousarray(v.transpose(0, 2, 1, 3)),
        "gamma": np.ascontiguousarray(gamma.transpose(0, 2, 1)),
        "beta": np.ascontiguousarray(beta.transpose(0, 2, 1)),
        "lam": regulariser(theta),
    }


def output_norm(o, weight, eps=1e-6):
    """Per-head RMSNorm of the layer's output (App. E): o [B, H, T, d_v], weight [H, d_v]
    -> y [B, T, H, d_v] = o / sqrt(mean(o^2) + eps) * weight[h]."""
    o, weight = _f64(o), _f64(weight)
    y = o / np.sqrt(np.mean(o * o, axis=-1, keepdims=True) + eps) * weight[None, :, None, :]
    return np.ascontiguousarray(y.transpose(0, 2, 1, 3))


def _silu_grad(u):
    s = sigmoid(u)
    return s * (1.0 + u * sigmoid(-_f64(u)))


def _short_conv_grad(x, w, du):
    """Gradients of short_conv: dx_t = sum_i w_i du_{t+i}, dw_i = sum_t du_t x_{t-i}."""
    T = x.shape[-2]
    dx, dw = np.zeros_like(x), np.zeros_like(_f64(w))
    for i in range(min(4, T)):
        dx[..., :T - i, :] += w[:, i] * du[..., i:, :]
        dw[:, i] = np.sum(du[..., i:, :] * x[..., :T - i, :], axis=tuple(range(x.ndim - 1)))
    return dx, dw


def frontend_backward(qp, kp, vp, conv_q, conv_k, conv_v, a_gamma, a_beta, theta, dq, dk, dv, dgamma, dbeta, dlam,
                      gamma_cap=0.9975, l2_eps=1e-6):
    """Gradients of frontend()'s inputs from those of its outputs, by the chain rule: a dict with
    dqp, dkp, dvp, dconv_q, dconv_k, dconv_v (None without conv_v), da_gamma, da_beta, dtheta."""
    out = {}
    for n, p, w, g in (("q", qp, conv_q, dq), ("k", kp, conv_k, dk), ("v", vp, conv_v, dv)):
        p, g = _f64(p), _f64(g).transpose(0, 2, 1, 3)
        B, T, H, d = p.shape
        if w is None:
            out["d" + n + "p"], out["dconv_" + n] = np.ascontiguousarray(g), None
            continue
        w = _f64(w)
        u = short_conv(p.reshape(B, T, H * d), w).reshape(B, T, H, d)
        if n != "v":
            f = silu(u)
            size = np.sqrt(np.sum(f * f, axis=-1, keepdims=True) + l2_eps)
            g = g / size - f * np.sum(f * g, axis=-1, keepdims=True) / size ** 3
        dp, dw = _short_conv_grad(p.reshape(B, T, H * d), w, (g * _silu_grad(u)).reshape(B, T, H * d))
        out["d" + n + "p"], out["dconv_" + n] = dp.reshape(B, T, H, d), dw
    open_, shut, beta = sigmoid(a_gamma), sigmoid(-_f64(a_gamma)), sigmoid(a_beta)
    dgamma, dbeta = _f64(dgamma).transpose(0, 2, 1), _f64(dbeta).transpose(0, 2, 1)
    cut = 1.0 - float(gamma_cap)
    out["da_gamma"] = dgamma * (1.0 - cut * beta ** 2) * open_ * shut
    out["da_beta"] = (dbeta - 2.0 * cut * dgamma * open_ * beta) * beta * sigmoid(-_f64(a_beta))
    out["dtheta"] = _f64(dlam) * sigmoid(theta)
    return out


def output_norm_backward(o, weight, dy, eps=1e-6):
    """Gradients of output_norm(): do [B, H, T, d_v], dweight [H, d_v] from dy [B, T, H, d_v]."""
    o, weight, dy = _f64(o), _f64(weight), _f64(dy).transpose(0, 2, 1, 3)
    size = np.sqrt(np.mean(o * o, axis=-1, keepdims=True) + eps)
    z = dy * weight[None, :, None, :]
    do = z / size - o * np.mean(z * o, axis=-1, keepdims=True) / size ** 3
    return do, np.sum(dy * o / size, axis=(0, 2))
