"""fp64 oracle of a language model's two ends: the scaled token embedding and the soft-capped softmax cross entropy over
a vocabulary, each with its gradient, written from the formulas (numpy).  A token or target outside [0, vocab) is none.

`cross_entropy_bounds` says how far a computation in fp32 with bf16 or fp32 operands may be off, element by element.
"""
import numpy as np


def embedding(table, tokens, scale=1.0):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for n, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[n] = scale * table[t]
    return out


def embedding_backward(tokens, dy, vocab, scale=1.0, base=None):
    """The table's gradient, and the sum of the magnitudes that were added and their number."""
    dy = np.asarray(dy, np.float64)
    grad = np.zeros((vocab, dy.shape[1]))
    size, count = np.zeros_like(grad), np.zeros((vocab, 1))
    for n, t in enumerate(tokens):
        if 0 <= t < vocab:
            grad[t] += scale * dy[n]
            size[t] += np.abs(scale * dy[n])
            count[t] += 1
    if base is not None:
        grad += np.asarray(base, np.float64)
    return grad, size, count


def counted(targets, vocab):
    t = np.asarray(targets)
    return (t >= 0) & (t < vocab)


def logits(h, table, cap):
    z = np.asarray(h, np.float64) @ np.asarray(table, np.float64).T
    return (cap * np.tanh(z / cap) if cap > 0 else z), z


def cross_entropy(h, table, targets, cap=0.0):
    l, z = logits(h, table, cap)
    top = l.max(axis=1)
    lse = top + np.log(np.exp(l - top[:, None]).sum(axis=1))
    there = counted(targets, table.shape[0])
    at = l[np.arange(len(l)), np.where(there, targets, 0)]
    return {"lse": lse, "loss": np.where(there, lse - at, 0.0), "best": z.argmax(axis=1)}


def cross_entropy_backward(h, table, targets, dloss, cap=0.0):
    h, table = np.asarray(h, np.float64), np.asarray(table, np.float64)
    l, _ = logits(h, table, cap)
    there = counted(targets, len(table))
    p = np.exp(l - cross_entropy(h, table, targets, cap)["lse"][:, None])
    y = np.zeros_like(p)
    y[there, np.asarray(targets)[there]] = 1.0
    dz = np.asarray(dloss, np.float64)[:, None] * (p - y)
    if cap > 0:
        dz *= 1.0 - (l / cap) ** 2
    dz[~there] = 0.0
    return {"dh": dz @ table, "dtable": dz[there].T @ h[there], "dz": dz, "p": p}


def cross_entropy_bounds(h, table, targets, dloss, cap, bf16):
    """Bounds on the errors of lse, loss, dh and dtable.  A product of D terms in fp32 is off by at most D 2^-23 of the sum
    of its terms' magnitudes (each addition by at most one unit in the last place, whichever way it rounds).  An fp32 factor
    may be held as two fp16 parts of its row scaled by a power of two to below 2^15.  The first has 11 bits, so what it
    leaves, a multiple of 2^-23 of the element's power of two, is at most 2^-11 of that: 12 bits, of which the second part
    keeps 11, off by one of those multiples at most, 2^-23.  Of an element below 2^-16 of the row's largest the second part
    is a multiple of 2^-24 of the scaled value, off by 2^-25: 2^-39 of the largest, which is 2^14 or more.  The product of
    two second parts, at most 2^-22, is left out.  Together 2 2^-23 + 2^-22 = 2^-21 of a term, and 2^-39 of the largest
    magnitude of either row times the other's sum.  The cap's tanh is good to 2^-20 of itself.  A sum of exponentials is good to 2^-18 (their
    arguments, up to about 20 where they weigh, are rounded at 2^-23 of themselves, and at most 128 additions follow each
    other), its logarithm to 2^-22 of itself.  What lies below fp32's smallest normal number, 2^-126, may be lost: a
    probability, and a gradient.  dz is rounded to bf16 (2^-8) for bf16 operands, and so are the gradients; but
    what rounding takes off the target's dz is added again (to 2^-23: an fp32 difference, and its product), and in
    the table's gradient of up to 1024 rows what it takes off any, itself rounded (2^-16)."""
    h, table = np.asarray(h, np.float64), np.asarray(table, np.float64)
    D, V, N = h.shape[1], len(table), len(h)
    l, _ = logits(h, table, cap)
    ah, at = np.abs(h), np.abs(table)
    dl = (D * 2.0 ** -23 + (0.0 if bf16 else 2.0 ** -21)) * (ah @ at.T) + 2.0 ** -20 * np.abs(l) * (cap > 0)
    if not bf16:
        dl += 2.0 ** -39 * (ah.max(axis=1)[:, None] * at.sum(axis=1) + ah.sum(axis=1)[:, None] * at.max(axis=1))
    ref = cross_entropy(h, table, targets, cap)
    dlse = dl.max(axis=1) + 2.0 ** -18 + 2.0 ** -22 * np.abs(ref["lse"])
    there = counted(targets, V)
    dat = dl[np.arange(N), np.where(there, targets, 0)]
    out = {"lse": dlse, "loss": np.where(there, dlse + dat + 2.0 ** -24 * np.abs(ref["loss"]), 0.0)}
    g = cross_entropy_backward(h, table, targets, dloss, cap)
    slope = 1.0 - (l / cap) ** 2 if cap > 0 else np.ones_like(l)
    # the slope moves by 2 |l| / cap^2 for a step of l
    dslope = 2.0 ** -20 * slope + (2.0 * np.abs(l) / cap ** 2 * dl if cap > 0 else 0.0)
    y = np.zeros_like(l)
    y[there, np.asarray(targets)[there]] = 1.0
    up = np.abs(np.asarray(dloss, np.float64))[:, None] * there[:, None]
    ddz = up * (slope * g["p"] * (dl + dlse[:, None] + 2.0 ** -18) + dslope * np.abs(g["p"] - y)) + np.abs(g["dz"]) * 2.0 ** -22
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    ddz += half * np.abs(g["dz"]) + 2.0 ** -126 * (up + 1.0 * there[:, None])
    size_h, size_e = np.abs(g["dz"]) @ np.abs(table), np.abs(g["dz"])[there].T @ np.abs(h[there])
    exact = ddz.copy()
    if bf16:
        exact[y == 1.0] -= (half - 2.0 ** -23) * np.abs(g["dz"][y == 1.0])
    few = ddz - (half - 2.0 ** -16) * np.abs(g["dz"]) if bf16 and N <= 1024 else exact
    out["dh"] = exact @ np.abs(table) + (V + 1) * 2.0 ** -23 * size_h + half * np.abs(g["dh"]) * 1.01 + 2.0 ** -126
    out["dtable"] = few[there].T @ np.abs(h[there]) + (2 * N + 1) * 2.0 ** -23 * size_e + half * np.abs(g["dtable"]) * 1.01 + 2.0 ** -126
    return out
