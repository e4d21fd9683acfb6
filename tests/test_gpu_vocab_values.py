"""The cross entropy's gradients where a row of the table is not finite: what does not count takes no part."""
import numpy as np
import pytest

from oracle import language_ends as E
from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _np(t):
    return t.double().cpu().numpy()


def _problem(rows, vocab, width, dtype, seed):
    rng = np.random.default_rng(seed)
    h = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda().to(dtype)
    table = torch.from_numpy((rng.standard_normal((vocab, width)) * width ** -0.5).astype(np.float32)).cuda().to(dtype)
    t = rng.integers(0, vocab, rows)
    up = rng.standard_normal(rows).astype(np.float32) / rows
    return h, table, t, torch.from_numpy(up).cuda()


# rows that are not a multiple of 64, and that are; some without a target or none; one piece of the table's depth and two
@pytest.mark.parametrize("rows,vocab,width,none", [(1, 50, 64, 0.0), (70, 200, 64, 0.0), (128, 300, 72, 0.3), (500, 777, 200, 0.1), (2100, 1201, 1800, 0.1)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_an_infinity_in_the_table(rows, vocab, width, none, cap):
    """Logits of -infinity, or -cap: neither has a gradient, so the table's is finite (0 in that row), although rows
    without a target, and those that fill up a step of the product, are zeros there, and 0 times infinity is not."""
    h, table, t, up = _problem(rows, vocab, width, BF16, rows)
    t[np.random.default_rng(1).random(rows) < none] = -1
    t[t == 7] = 8
    h[:, 3] = h[:, 3].abs() + 0.5
    table[7, 3] = -float("inf")
    targets = torch.from_numpy(t).cuda()
    f = L.cross_entropy(h, table, targets, cap=cap)
    got = _np(L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap, want_dh=False)["dtable"])
    # the reference holds a far finite number in its place: exp(l) is 0, or the slope at -cap is, to fp32's last place
    away = _np(table)
    away[7] = 0.0
    away[7, 3] = -1e4
    want, bound = E.cross_entropy_backward(_np(h), away, t, _np(up), cap), E.cross_entropy_bounds(_np(h), away, t, _np(up), cap, True)
    keep = np.arange(vocab) != 7
    assert np.isfinite(got).all() and not got[7].any()
    # that far row's own product, exact here, is not to widen the bounds of the others
    near = E.cross_entropy_bounds(_np(h), np.where(keep[:, None], away, 0.0), t, _np(up), cap, True)["dtable"]
    assert (np.abs(got - want["dtable"]) <= np.minimum(bound["dtable"], near * 1.01 + 1e-30))[keep].all()


@pytest.mark.parametrize("rows", [20, 70, 1500])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_row_counts(rows, dtype):
    """Whatever the table and the rows hold, the gradients are zeros."""
    h, table, t, up = _problem(rows, 300, 64, dtype, rows)
    table[5], table[6], table[7, 1] = float("nan"), float("inf"), -float("inf")
    h[3] = float("nan")
    targets = torch.full((rows,), -1, device="cuda")
    g = L.cross_entropy_backward(h, table, targets, torch.full((rows,), float("nan"), device="cuda"), up, cap=30.0)
    assert all(bool((x == 0).all()) for x in g.values())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_nan_in_the_table_of_rows_that_count(dtype):
    """Every logit's sum meets it: so do the gradients, as the formula says."""
    h, table, t, up = _problem(70, 100, 64, dtype, 2)
    table[9, 2] = float("nan")
    targets = torch.from_numpy(t).cuda()
    f = L.cross_entropy(h, table, targets, cap=30.0)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0)
    assert bool(f["lse"].isnan().all()) and bool(g["dh"].isnan().all()) and bool(g["dtable"].isnan().all())


@pytest.mark.parametrize("rows", [1, 32, 33, 64, 200])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_one_channel_far_above_the_others(rows, cap):
    """fp32 rows with a channel 2^30 times the others, which the table does not take.  Up to 32 rows, of three parts each, every
    product is good to 2^-23 of itself; more are held in two parts of 11 bits below their row's largest magnitude, so the
    others may be off by 2^-39 of that: 2^-9 of themselves here."""
    h, table, t, up = _problem(rows, 300, 96, F32, rows)
    h[:, 5], table[:, 5] = 2.0 ** 30, 0.0
    f = L.cross_entropy(h, table, torch.from_numpy(t).cuda(), cap=cap)
    g = L.cross_entropy_backward(h, table, torch.from_numpy(t).cuda(), f["lse"], up, cap=cap)
    held = _np(h)
    if rows <= 32:
        held[:, 5] = 0.0      # it takes no part in the bounds
    want, grads = E.cross_entropy(_np(h), _np(table), t, cap), E.cross_entropy_backward(_np(h), _np(table), t, _np(up), cap)
    bound = E.cross_entropy_bounds(held, _np(table), t, _np(up), cap, False)
    for n, got, ref in (("lse", f["lse"], want["lse"]), ("loss", f["loss"], want["loss"]), ("dh", g["dh"], grads["dh"])):
        assert (np.abs(_np(got) - ref) <= bound[n]).all(), n
    keep = np.arange(96) != 5
    assert (np.abs(_np(g["dtable"]) - grads["dtable"]) <= bound["dtable"])[:, keep].all()
    # and the same rows among more: to the sum of both bounds
    if rows == 32:
        more = L.cross_entropy(torch.cat([h, h]), table, torch.from_numpy(np.concatenate([t, t])).cuda(), cap=cap)
        wide = E.cross_entropy_bounds(_np(h), _np(table), t, _np(up), cap, False)
        assert (np.abs(_np(more["lse"][:32]) - _np(f["lse"])) <= wide["lse"] + bound["lse"]).all()
