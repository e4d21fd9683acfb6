"""Sizes that between them take every tile, layer and piece of the cross entropy's products, with the plan that each of
them is here for (tests/test_vocab_plan.py holds the plans, tests/test_gpu_vocab_tiles.py runs the sizes), and the
oracle's results and bounds for sizes that are too much for it: the same formulas, some rows at a time, on the device."""
import numpy as np

try:
    import torch
except ImportError:      # the plans alone need none
    torch = None

F32, BF16 = 0, 1
# rows, vocabulary, width, type; the tile of the forward's logits, of dz, of dh and of the table's gradient (wide,
# middle, narrow, thin), the last two with their layers.  Odd sizes, so that every tile has a remainder, and three steps
# of k or more but where one row of h makes a step.
TILES = [
    (3, 200, 200, BF16, "T", "T", "T1", "N1"),
    (3, 16003, 321, BF16, "T", "T", "T28", "M1"),
    (33, 5003, 2050, BF16, "N", "N", "N9", "W1"),
    (777, 200, 200, BF16, "N", "N", "N1", "N3"),
    (70, 16003, 2050, BF16, "N", "N", "M28", "W1"),
    (6001, 200, 1000, BF16, "N", "N", "M1", "N9"),
    (3001, 200, 4097, BF16, "N", "N", "W1", "M6"),
    (6001, 777, 200, BF16, "M", "M", "N1", "N13"),
    (2049, 5003, 200, BF16, "W", "W", "N4", "M6"),
    (4100, 777, 2050, BF16, "N", "N", "W1", "N1"),
    (1100, 9001, 1000, BF16, "W", "W", "M6", "W1"),
    (4100, 6001, 768, BF16, "W", "W", "W4", "W3"),
    (3, 1201, 200, F32, "T", "T", "N2", "N1"),
    (31, 20011, 257, F32, "T", "T", "N28", "W1"),
    (70, 200, 200, F32, "N", "N", "N1", "N1"),
    (70, 9001, 321, F32, "N", "N", "N13", "M1"),
    (70, 20011, 1000, F32, "M", "M", "M28", "W1"),
    (2049, 200, 1500, F32, "N", "N", "M1", "N4"),
    (1500, 200, 4097, F32, "N", "N", "W1", "M3"),
    (777, 5003, 768, F32, "W", "W", "M6", "M1"),
    (2049, 5003, 257, F32, "M", "M", "N3", "W4"),
    (3001, 2003, 520, F32, "W", "W", "W4", "M3"),
]

# rows, vocabulary, width, type; the parts of the table that the forward copies one after the other, and the pieces of
# the vocabulary that the gradients take: both of the last kind shorter than the others
PIECES = [
    (3, 140001, 1000, BF16, 2, 1),       # a copied table, rows of 1000 channels
    (1000, 70000, 64, BF16, 1, 2),       # dz with all of its rounding's rest behind it
    (9000, 16000, 40, BF16, 1, 2),       # the targets' rests, from sorted targets
    (17000, 9001, 32, BF16, 1, 2),       # the same over runs of sorted rows
    (16384, 9000, 2048, BF16, 1, 2),     # wide tiles, no layers
    (40, 70000, 2048, F32, 3, 2),        # planes and exponents of a table that is copied
    (20, 100000, 2048, F32, 1, 2),       # few rows, which read it as it lies for the logits
    (16384, 8500, 24, F32, 1, 2),        # layers of dh, added to by the second piece
    (4100, 40001, 300, F32, 1, 2),       # wide tiles
]


def reference(h, table, targets, up, cap, keeps_all):
    """lse, loss, best, dh and dtable in 64 bits and, as oracle.language_ends.cross_entropy_bounds has them, their bounds
    (keeps_all: all that dz's rounding to bf16 takes off is in the table's gradient, not the targets' alone)."""
    bf16 = h.dtype is torch.bfloat16
    N, (V, D) = h.shape[0], table.shape
    w = table.double()
    aw, wt = w.abs(), w.t().contiguous()
    at = aw.t().contiguous()
    out = {n: [] for n in ("lse", "loss", "best", "dh")}
    bound = {n: [] for n in ("lse", "loss", "dh")}
    dtable, few_sum, size_e = (torch.zeros_like(w) for _ in range(3))
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    step = max(1, (1 << 25) // V)
    for lo in range(0, N, step):
        x, t, u = h[lo:lo + step].double(), targets[lo:lo + step].long(), up[lo:lo + step].double()
        n = torch.arange(x.shape[0], device=x.device)
        there = (t >= 0) & (t < V)
        pick = torch.where(there, t, 0)
        z = x @ wt
        l = cap * torch.tanh(z / cap) if cap > 0 else z
        slope = 1.0 - (l / cap) ** 2 if cap > 0 else torch.ones_like(l)
        lse = torch.logsumexp(l, dim=1)
        out["best"].append(z.argmax(dim=1))
        out["lse"].append(lse)
        loss = torch.where(there, lse - l[n, pick], 0.0)
        out["loss"].append(loss)
        dl = (D * 2.0 ** -23 + (0.0 if bf16 else 2.0 ** -21)) * (x.abs() @ at) + (2.0 ** -20 * l.abs() if cap > 0 else 0.0)
        if not bf16:
            dl += 2.0 ** -39 * (x.abs().amax(dim=1)[:, None] * aw.sum(dim=1) + x.abs().sum(dim=1)[:, None] * aw.amax(dim=1))
        dlse = dl.amax(dim=1) + 2.0 ** -18 + 2.0 ** -22 * lse.abs()
        bound["lse"].append(dlse)
        bound["loss"].append(torch.where(there, dlse + dl[n, pick] + 2.0 ** -24 * loss.abs(), 0.0))
        p = torch.exp(l - lse[:, None])
        weight = (u.abs() * there)[:, None]
        dz = p.clone()
        dz[n, pick] -= there.double()
        ddz = weight * (slope * p * (dl + dlse[:, None] + 2.0 ** -18)
                        + (2.0 ** -20 * slope + (2.0 * l.abs() / cap ** 2 * dl if cap > 0 else 0.0)) * dz.abs())
        dz = torch.where(there[:, None], dz * slope * u[:, None], 0.0)
        size = dz.abs()
        ddz += size * 2.0 ** -22 + half * size + 2.0 ** -126 * (weight + 1.0 * there[:, None])
        exact = ddz.clone()
        if bf16:
            exact[n, pick] -= torch.where(there, (half - 2.0 ** -23) * size[n, pick], 0.0)
        few = ddz - (half - 2.0 ** -16) * size if bf16 and keeps_all else exact
        dh = dz @ w
        out["dh"].append(dh)
        bound["dh"].append(exact @ aw + (V + 1) * 2.0 ** -23 * (size @ aw) + half * dh.abs() * 1.01 + 2.0 ** -126)
        x = torch.where(there[:, None], x, 0.0)
        dtable += dz.t().contiguous() @ x
        few_sum += torch.where(there[:, None], few, 0.0).t().contiguous() @ x.abs()
        size_e += size.t().contiguous() @ x.abs()
    out = dict({n: torch.cat(v) for n, v in out.items()}, dtable=dtable)
    bound = {n: torch.cat(v) for n, v in bound.items()}
    bound["dtable"] = few_sum + (2 * N + 1) * 2.0 ** -23 * size_e + half * dtable.abs() * 1.01 + 2.0 ** -126
    return out, bound


def problem(rows, vocab, width, dtype, seed, device="cuda"):
    """Rows that lean towards their target, one in ten of them without one."""
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == BF16 else torch.float32
    table = torch.from_numpy((rng.standard_normal((vocab, width)) * width ** -0.5).astype(np.float32)).to(device).to(dt)
    t = np.minimum((np.exp(rng.random(rows) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1)
    t[rng.random(rows) < 0.1] = rng.choice([-1, vocab])
    t[0] = vocab - 1
    targets = torch.from_numpy(t).to(device)
    lean = torch.from_numpy((rng.random((rows, 1)) * 8).astype(np.float32)).to(device)
    h = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).to(device)
    h = (h + lean * table[torch.where((targets >= 0) & (targets < vocab), targets, 0)].float()).to(dt)
    up = torch.from_numpy((rng.standard_normal(rows) / rows).astype(np.float32)).to(device)
    return h, table, targets, up
