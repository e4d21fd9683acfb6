"""The token embedding, the cross entropy over a vocabulary and their gradients against the fp64 oracle.

Tolerances, element by element.  A look-up is one product rounded once: half a step of the result's type (2^-24 of the
value in fp32, 2^-8 in bf16) on top of the product's 2^-24.  A sum of n rows is off by at most n 2^-24 of the sum of their
magnitudes, and is scaled, added to the base and rounded once each.  Those of the cross entropy are
oracle/language_ends.py's cross_entropy_bounds.
"""
import numpy as np
import pytest

from oracle import language_ends as E
from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _np(t):
    return t.double().cpu().numpy()


def _within(got, want, bound, name):
    got = _np(got)
    assert got.shape == want.shape and np.isfinite(got).all(), name
    worst = np.abs(got - want) / np.maximum(bound, 1e-300)
    assert (np.abs(got - want) <= bound).all(), (name, float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))


def _tokens(rng, rows, vocab, wide=True, none=0.1):
    t = np.minimum((np.exp(rng.random(rows) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1)
    odd = rng.random(rows) < none
    t[odd] = rng.choice([-1, -100, vocab, vocab + 7], odd.sum())
    return t, torch.from_numpy(t if wide else t.astype(np.int32)).cuda()


def _table(rng, rows, width, dtype, pad=0, scale=1.0, shift=0):
    """Rows of width that lie width + pad apart, from element `shift` of an allocation on."""
    stride = width + pad
    flat = torch.zeros(rows * stride + shift + 8, dtype=dtype, device="cuda")
    x = flat[shift:shift + rows * stride].view(rows, stride)[:, :width]
    x.copy_(torch.from_numpy((rng.standard_normal((rows, width)) * scale).astype(np.float32)))
    return x


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("rows,vocab,width,pad,shift", [
    (1, 1, 1, 0, 0), (1, 50, 2048, 0, 0), (3, 7, 8, 0, 0), (100, 1000, 64, 0, 0), (257, 33, 321, 0, 0), (40, 100, 96, 32, 0),
    (40, 100, 96, 5, 0), (40, 100, 64, 0, 3), (5000, 301, 40, 0, 0), (300, 64, 5000, 0, 0)])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_embedding(rows, vocab, width, pad, shift, dtype, out):
    rng = np.random.default_rng(rows + width)
    table = _table(rng, vocab, width, dtype, pad, shift=shift)
    t, tokens = _tokens(rng, rows, vocab, wide=rows % 2 == 0)
    got = L.embedding(table, tokens, scale=1.7, out_dtype=out)
    scale = float(np.float32(1.7))
    want = E.embedding(_np(table), t, scale)
    _within(got, want, np.abs(want) * (HALF[out] + 2.0 ** -24) * 1.001, "embedding")
    assert bool((got[torch.from_numpy(~E.counted(t, vocab)).cuda()] == 0).all())
    # into spaced rows, whose gaps stay as they were
    room = torch.full((rows, width + 3), 7.0, dtype=out, device="cuda")
    assert L.embedding(table, tokens, scale=1.7, out=room[:, :width]) is not None
    assert torch.equal(room[:, :width], got) and bool((room[:, width:] == 7).all())


def test_embedding_shapes_and_values():
    """Tokens of any shape; what a row without a token would read is not looked at; a NaN of the table stays one."""
    table = torch.full((4, 16), float("nan"), device="cuda")
    table[2] = 3.0
    tokens = torch.tensor([[2, -1], [9, 2]], device="cuda")
    got = L.embedding(table, tokens, scale=2.0)
    assert got.shape == (2, 2, 16) and bool((got[0, 0] == 6).all()) and bool((got[0, 1] == 0).all()) and bool((got[1, 0] == 0).all())
    assert bool(L.embedding(table, tokens * 0).isnan().all())
    assert L.embedding(table, tokens[:0]).shape == (0, 2, 16)


# ------------------------------------------------------------------ its gradient
@pytest.mark.parametrize("rows,vocab,width,pad", [
    (1, 1, 1, 0), (1, 5003, 64, 0), (33, 1, 8, 0), (64, 3, 40, 0), (777, 5003, 321, 0), (2048, 50, 64, 0), (2049, 50, 64, 8),
    (2100, 600, 72, 3), (5000, 300, 16, 0), (9000, 70000, 8, 0), (3000, 2, 24, 0), (70, 140000, 4, 0), (4100, 270000, 8, 0),
    (16384, 40, 8, 0), (16385, 1000, 8, 0), (40000, 300, 9, 1)])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
def test_embedding_backward(rows, vocab, width, pad, dtype, out):
    rng = np.random.default_rng(rows + vocab)
    t, tokens = _tokens(rng, rows, vocab, wide=rows % 2 == 0)
    dy = _table(rng, rows, width, dtype, pad)
    dy[torch.from_numpy(~E.counted(t, vocab)).cuda()] = float("nan")       # rows without a token are not read
    scale = float(np.float32(0.3))
    clean = np.where(E.counted(t, vocab)[:, None], _np(dy), 0.0)
    want, size, count = E.embedding_backward(t, clean, vocab, scale)
    bound = (count + 2) * 2.0 ** -24 * size * 1.001 + HALF[out] * np.abs(want) * 1.001
    got = L.embedding_backward(tokens, dy, vocab, scale=0.3, grad_dtype=out)
    _within(got, want, bound, "gradient")
    assert bool((got[torch.from_numpy(count[:, 0] == 0).cuda()] == 0).all())
    assert torch.equal(got, L.embedding_backward(tokens, dy, vocab, scale=0.3, grad_dtype=out))
    # added to what is there; rows of other tokens are not touched, nor the gaps between spaced rows
    room = torch.full((vocab, width + pad), 7.0, dtype=out, device="cuda")
    room[:, :width] = torch.from_numpy(rng.standard_normal((vocab, width))).to(out)
    base = room.clone()
    want, size, count = E.embedding_backward(t, clean, vocab, scale, _np(base[:, :width]))
    total = size + np.abs(_np(base[:, :width]))
    L.embedding_backward(tokens, dy, vocab, scale=0.3, out=room[:, :width], accumulate=True)
    _within(room[:, :width], want, (count + 3) * 2.0 ** -24 * total * 1.001 + HALF[out] * np.abs(want) * 1.001, "accumulated")
    quiet = torch.from_numpy(count[:, 0] == 0).cuda()
    assert torch.equal(room[quiet], base[quiet]) and torch.equal(room[:, width:], base[:, width:])


@pytest.mark.parametrize("rows", [7, 8, 9, 15, 16, 17, 511, 512, 513, 3000, 5000, 8191, 8192, 8193, 16384, 16385, 17000, 33793, 40000])
def test_one_token_everywhere(rows):
    """Every row the same token, at lengths around whole pieces of 8 and 16 and runs of 512 sorted positions."""
    rng = np.random.default_rng(rows)
    dy = _table(rng, rows, 40, F32)
    t = np.full(rows, 2)
    got = L.embedding_backward(torch.from_numpy(t).cuda(), dy, 4)
    want, size, count = E.embedding_backward(t, _np(dy), 4)
    _within(got, want, (count + 2) * 2.0 ** -24 * size, "gradient")


def test_embedding_backward_without_rows():
    out = torch.full((5, 12), 3.0, device="cuda")
    none, dy = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros((0, 12), device="cuda")
    L.embedding_backward(none, dy, 5, out=out, accumulate=True)
    assert bool((out == 3).all())
    L.embedding_backward(none, dy, 5, out=out)
    assert bool((out == 0).all())
    nothing = torch.full((70,), -1, device="cuda")
    assert bool((L.embedding_backward(nothing, torch.full((70, 12), float("nan"), device="cuda"), 5) == 0).all())


# ------------------------------------------------------------------ cross entropy
def _problem(rows, vocab, width, dtype, seed, pad=0, shift=0, none=0.1, size=1.0):
    rng = np.random.default_rng(seed)
    h = _table(rng, rows, width, dtype, pad, size, shift)
    table = _table(rng, vocab, width, dtype, pad, width ** -0.5, shift)
    t, targets = _tokens(rng, rows, vocab, wide=rows % 2 == 0, none=none)
    # leaning towards the target, so that losses are of every size
    lean = (rng.random(rows) * 8 * E.counted(t, vocab)).astype(np.float32)
    h += (torch.from_numpy(lean).cuda()[:, None] * table[torch.from_numpy(np.where(E.counted(t, vocab), t, 0)).cuda()].float()).to(dtype)
    up = rng.standard_normal(rows).astype(np.float32) / rows
    return h, table, t, targets, torch.from_numpy(up).cuda()


def _check_all(h, table, t, targets, up, cap):
    nh, nt, nu = _np(h), _np(table), _np(up)
    bf16 = h.dtype is BF16
    want, grads = E.cross_entropy(nh, nt, t, cap), E.cross_entropy_backward(nh, nt, t, nu, cap)
    bound = E.cross_entropy_bounds(nh, nt, t, nu, cap, bf16)
    f = L.cross_entropy(h, table, targets, cap=cap, want_best=True)
    for n in ("lse", "loss"):
        _within(f[n], want[n], bound[n], n)
    # the largest product, within what its terms' rounding may hide
    z = nh @ nt.T
    slack = 2.0 * (nh.shape[1] + 4) * 2.0 ** -23 * (np.abs(nh) @ np.abs(nt).T).max(axis=1)      # as cross_entropy_bounds has it
    best = f["best"].cpu().numpy()
    assert (z[np.arange(len(z)), best] >= z.max(axis=1) - slack).all()
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap)
    for n in ("dh", "dtable"):
        _within(g[n], grads[n], bound[n], n)
    again = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap, want_dh=False)
    assert set(again) == {"dtable"} and torch.equal(again["dtable"], g["dtable"])
    again = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap, want_dtable=False)
    assert set(again) == {"dh"} and torch.equal(again["dh"], g["dh"])
    return f, g


SIZES = [(1, 1, 1), (1, 5003, 64), (32, 300, 128), (3, 200, 129), (20, 130, 383), (2, 50, 2048), (5, 64, 8), (16, 63, 65), (31, 65, 100), (33, 129, 64), (64, 300, 200), (65, 257, 321),
         (100, 5003, 321), (130, 1000, 128), (300, 777, 72), (513, 513, 64)]


@pytest.mark.parametrize("rows,vocab,width", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cap", [0.0, 30.0, 2.0])
def test_cross_entropy(rows, vocab, width, dtype, cap):
    _check_all(*_problem(rows, vocab, width, dtype, seed=rows + width), cap)


@pytest.mark.parametrize("pad,shift", [(8, 0), (64, 8), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_cross_entropy_of_spaced_and_unaligned_rows(pad, shift, dtype):
    h, table, t, targets, up = _problem(70, 200, 128, dtype, 5, pad, shift)
    f, g = _check_all(h, table, t, targets, up, 30.0)
    dense = L.cross_entropy(h.contiguous().clone(), table.contiguous().clone(), targets, cap=30.0)
    assert torch.equal(dense["lse"], f["lse"]) and torch.equal(dense["loss"], f["loss"])


@pytest.mark.parametrize("rows,vocab,width,dtype", [
    (4096, 3700, 64, BF16),        # the widest tiles, logits
    (2048, 2000, 1900, BF16),      # and the gradients', ragged
    (16384, 8500, 24, BF16),       # two pieces of the vocabulary
    (6000, 8200, 16, F32),         # the same with three planes
    (3000, 200, 40, F32), (40, 9000, 40, BF16), (700, 90, 30, BF16),    # few tiles: the sums are cut into layers
    (1024, 301, 72, BF16), (1025, 301, 72, BF16)])      # the most rows whose dz has its rounding's rest behind it, and one more
def test_cross_entropy_of_larger_sizes(rows, vocab, width, dtype):
    _check_all(*_problem(rows, vocab, width, dtype, seed=rows), 30.0)


def test_products_far_past_a_copied_piece():
    """A table that is copied in several pieces: fp32 rows of 2048 channels, 64 MiB of planes at a time."""
    h, table, t, targets, up = _problem(20, 6000, 2048, F32, 3)
    f = L.cross_entropy(h, table, targets, cap=30.0, want_best=True)
    want, bound = E.cross_entropy(_np(h), _np(table), t, 30.0), E.cross_entropy_bounds(_np(h), _np(table), t, _np(up), 30.0, False)
    for n in ("lse", "loss"):
        _within(f[n], want[n], bound[n], n)
    assert (f["best"].cpu().numpy() == want["best"]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_do_not_count(dtype):
    """NaN and infinity in rows without a target, in their lse and dloss: no other row and no gradient sees them."""
    h, table, t, targets, up = _problem(150, 300, 64, dtype, 9, none=0.3)
    f = L.cross_entropy(h, table, targets, cap=30.0)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0)
    away = torch.from_numpy(~E.counted(t, 300)).cuda()
    bad = h.clone()
    bad[away] = float("nan")
    bad[away.nonzero()[0]] = float("inf")
    fb = L.cross_entropy(bad, table, targets, cap=30.0)
    lse, upb = f["lse"].clone(), up.clone()
    lse[away], upb[away] = float("nan"), float("inf")
    gb = L.cross_entropy_backward(bad, table, targets, lse, upb, cap=30.0)
    assert torch.equal(fb["loss"], f["loss"]) and bool((f["loss"][away] == 0).all()) and torch.equal(fb["lse"][~away], f["lse"][~away])
    assert torch.equal(gb["dh"], g["dh"]) and torch.equal(gb["dtable"], g["dtable"]) and bool((g["dh"][away] == 0).all())
    none = torch.full_like(targets, -1)
    fn = L.cross_entropy(bad, table, none, cap=30.0)
    gn = L.cross_entropy_backward(bad, table, none, lse, upb, cap=30.0)
    assert bool((fn["loss"] == 0).all()) and bool((gn["dh"] == 0).all()) and bool((gn["dtable"] == 0).all())


def test_values_that_are_not_finite():
    h, table, t, targets, up = _problem(40, 100, 64, BF16, 11, none=0.0)
    table[7, 3] = float("nan")
    f = L.cross_entropy(h, table, targets, cap=30.0, want_best=True)
    assert bool(f["lse"].isnan().all()) and bool(f["loss"].isnan().all())
    table[7] = -h[0] * float("inf")       # a product of -infinity for row 0: capped, or no weight at all
    h0 = h[:1].contiguous()
    assert bool(L.cross_entropy(h0, table, cap=30.0)["lse"].isfinite().all())
    got = L.cross_entropy(h0, table)["lse"]
    keep = torch.cat([table[:7], table[8:]])
    want = np.log(np.exp(_np(h0) @ _np(keep).T).sum())
    assert abs(float(got) - want) < 1e-4


def test_ends_of_fp32():
    """Products of 2^120 by 2^-120 and far logits without a cap; fp32 values whose nearest bf16 is an infinity."""
    rng = np.random.default_rng(4)
    h = torch.from_numpy((rng.standard_normal((10, 64)) * 2.0 ** 100).astype(np.float32)).cuda()
    table = torch.from_numpy((rng.standard_normal((90, 64)) * 2.0 ** -100).astype(np.float32)).cuda()
    h[0] = 3.4e38
    table[:, :] = torch.where(table.abs() < 2.0 ** -126, 2.0 ** -126, table)
    targets = torch.arange(10, device="cuda")
    f = L.cross_entropy(h[1:].contiguous(), table, targets[1:].contiguous())
    want = E.cross_entropy(_np(h[1:]), _np(table), np.arange(1, 10))
    bound = E.cross_entropy_bounds(_np(h[1:]), _np(table), np.arange(1, 10), np.ones(9), 0.0, False)
    for n in ("lse", "loss"):
        _within(f[n], want[n], bound[n], n)
    f = L.cross_entropy(h[:1].contiguous(), table * 2.0 ** -25, targets[:1].contiguous())
    nt = _np(table * 2.0 ** -25)
    want = E.cross_entropy(_np(h[:1]), nt, [0])
    bound = E.cross_entropy_bounds(_np(h[:1]), nt, [0], np.ones(1), 0.0, False)
    # parts of the table below fp32's normal range may be dropped: 64 products of at most 2^-126 by 2^128
    extra = 64 * 2.0 ** -126 * 2.0 ** 128
    _within(f["lse"], want["lse"], bound["lse"] + extra, "lse")
    # logits in the hundreds
    big = torch.from_numpy((rng.standard_normal((10, 64)) * 100).astype(np.float32)).cuda()
    one = torch.from_numpy(rng.standard_normal((90, 64)).astype(np.float32)).cuda()
    _check_all(big, one, np.arange(10), targets, torch.ones(10, device="cuda"), 0.0)
    _check_all(big, one, np.arange(10), targets, torch.ones(10, device="cuda"), 30.0)


def test_ties_go_to_the_lowest():
    h = torch.ones((70, 64), dtype=BF16, device="cuda")
    table = torch.ones((1000, 64), dtype=BF16, device="cuda")
    table[300] = table[299] = table[900] = 2.0
    assert bool((L.cross_entropy(h, table, want_best=True)["best"] == 299).all())
    assert bool((L.cross_entropy(h * 0, table, want_best=True)["best"] == 0).all())
    assert bool((L.cross_entropy(h * float("nan"), table, want_best=True)["best"] == -1).all())


def test_no_rows():
    table = torch.randn((30, 64), device="cuda")
    none, t = torch.zeros((0, 64), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    f = L.cross_entropy(none, table, t, cap=1.0, want_best=True)
    assert f["loss"].shape == f["lse"].shape == f["best"].shape == (0,)
    g = L.cross_entropy_backward(none, table, t, f["lse"], f["lse"], cap=1.0)
    assert g["dh"].shape == (0, 64) and bool((g["dtable"] == 0).all())


def test_leading_dimensions():
    h, table, t, targets, up = _problem(24, 100, 64, BF16, 2)
    flat = L.cross_entropy(h, table, targets, cap=30.0, want_best=True)
    f = L.cross_entropy(h.view(2, 3, 4, 64), table, targets.view(2, 3, 4), cap=30.0, want_best=True)
    assert all(torch.equal(f[n].view(-1), flat[n]) and f[n].shape == (2, 3, 4) for n in flat)
    g = L.cross_entropy_backward(h.view(2, 3, 4, 64), table, targets.view(2, 3, 4), f["lse"], up.view(2, 3, 4), cap=30.0)
    assert g["dh"].shape == (2, 3, 4, 64)


@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_small_losses(cap):
    """Rows that are sure of their target: the loss, and the target's 1 - p, are the small difference of two numbers near
    12.  Rows of one 1 make the products exact, and each gradient one element of dz.  The sum over 50 rows of the table in
    units of the target's exponential takes 8 additions a lane, 2 between lanes and 1 between waves, of 2^-24 each, two
    exponentials of 2^-23 each: 16 2^-24 in all; the others' part, about the loss, is good to 2^-18 and moves with tanh's
    2^-20 of two logits.  lse is rounded once, 2^-24 of itself, before the gradient takes it."""
    rng = np.random.default_rng(12)
    rows, vocab, width = 40, 50, 64
    nt = rng.standard_normal((vocab, width)).astype(np.float32)
    t = rng.integers(0, vocab, rows)
    nt[t, np.arange(rows)] = 10.0 + 4.0 * rng.random(rows)
    h, table = torch.eye(rows, width, device="cuda"), torch.from_numpy(nt).cuda()
    targets, up = torch.from_numpy(t).cuda(), torch.ones(rows, device="cuda")
    f = L.cross_entropy(h, table, targets, cap=cap)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap)
    nh = np.eye(rows, width)
    want = E.cross_entropy(nh, nt, t, cap)
    assert want["loss"].max() < 0.1 and want["loss"].min() > 1e-6
    top = np.abs(want["lse"]).max()
    bound = 16 * 2.0 ** -24 + want["loss"] * (2.0 ** -18 + 2.0 ** -19 * top)
    _within(f["loss"], want["loss"], bound, "loss")
    assert bool((f["loss"] > 0).all())
    dz = E.cross_entropy_backward(nh, nt, t, np.ones(rows), cap)["dz"][np.arange(rows), t]
    got = g["dtable"][targets, torch.arange(rows, device="cuda")]
    _within(got, dz, bound + 2.0 ** -24 * top + 2.0 ** -22 + 2.0 ** -20 * np.abs(dz), "dz")


def test_gradients_against_differences():
    """Central differences of the forward in fp32: a step of 2^-6 leaves the forward's own rounding (about 2e-6 of a loss
    of 5) at 2e-4 of a slope, and the third derivative at less than that."""
    h, table, t, targets, up = _problem(6, 40, 64, F32, 8, none=0.0)
    up = torch.ones_like(up)
    g = L.cross_entropy_backward(h, table, targets, L.cross_entropy(h, table, targets, cap=5.0)["lse"], up, cap=5.0)
    rng = np.random.default_rng(0)
    step = 2.0 ** -6
    for name, x in (("dh", h), ("dtable", table)):
        for _ in range(10):
            way = torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)).cuda()
            way /= way.norm()
            ends = [L.cross_entropy(*((x + s * way, table) if name == "dh" else (h, x + s * way)), targets, cap=5.0)["loss"].double().sum()
                    for s in (step, -step)]
            slope = float(ends[0] - ends[1]) / (2 * step)
            assert abs(slope - float((g[name].double() * way.double()).sum())) < 2e-3, name
