"""What rounding dz to bf16 costs the gradients: next to nothing where the rows' targets are the large elements of dz.

Its other elements are the probabilities.  Where those are spread over the table, an element of dz other than the
target's is far below it, and each gradient is then off by its own rounding alone: the norm of its error is that of
the exact gradient rounded to bf16, to the accuracy of a norm over as many roundings."""
import numpy as np
import pytest

from oracle import language_ends as E
from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _np(t):
    return t.double().cpu().numpy()


def _problem(rows, vocab, width, seed, spread):
    """Logits of about one, targets as frequent as in text (spread) or all of a few."""
    rng = np.random.default_rng(seed)
    h = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda().to(BF16)
    table = torch.from_numpy((rng.standard_normal((vocab, width)) * width ** -0.5).astype(np.float32)).cuda().to(BF16)
    t = np.minimum((np.exp(rng.random(rows) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1) if spread else rng.integers(0, 3, rows)
    t[rng.random(rows) < 0.05] = -1
    t[0], t[1] = vocab - 1, -1
    up = (rng.random(rows) + 0.5).astype(np.float32) / rows
    return h, table, t, torch.from_numpy(t).cuda(), torch.from_numpy(up).cuda()


# All of dz's rounding is kept for up to 1024 rows, or 4.3e9 products; else the targets' is: sorted by one launch (2048 rows)
# and by more, summed in pieces of 8 sorted rows (8192) and of 16, over runs of pieces (16384), one channel or eight (2^22
# values) a lane; with tables of one piece and of several (2^27 elements of dz)
@pytest.mark.parametrize("rows,vocab,width,spread", [
    (1000, 3000, 64, True), (1025, 3000, 64, True), (1500, 900, 7, True), (17000, 700, 24, False),
    (2048, 3001, 720, True), (2049, 3001, 721, True), (4100, 2003, 1024, True), (1100, 130000, 40, True), (9000, 16000, 40, True),
    (9001, 1000, 520, True), (17000, 9001, 32, True), (17000, 1100, 300, False), (1600, 700000, 4, True)])
def test_gradients_are_off_by_their_own_rounding(rows, vocab, width, spread):
    h, table, t, targets, up = _problem(rows, vocab, width, rows + width, spread)
    f = L.cross_entropy(h, table, targets, cap=30.0)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0)
    # the definition in 64 bits, some rows at a time
    w, dh, dtable = table.double(), [], torch.zeros((vocab, width), dtype=torch.float64, device="cuda")
    there = (targets >= 0).double()
    for lo in range(0, rows, 1000):
        x, m = h[lo:lo + 1000].double(), slice(lo, lo + 1000)
        y = torch.tanh(x @ w.t().contiguous() / 30.0)
        dz = torch.softmax(30.0 * y, dim=1)
        dz[torch.arange(len(x), device="cuda"), targets[m].clamp(min=0)] -= 1.0
        dz *= (1.0 - y * y) * (up[m].double() * there[m])[:, None]
        dh.append(dz @ w)
        dtable += dz.t().contiguous() @ x
    for name, want in (("dh", torch.cat(dh)), ("dtable", dtable)):
        off, own = float((g[name].double() - want).norm()), float((want.to(BF16).double() - want).norm())
        # some 10^4 roundings or more: their norms differ by a percent or two; without the rests the ratio is 1.2 and more
        assert off <= 1.05 * own, (name, off / own)
    again = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0, want_dh=False)
    assert torch.equal(again["dtable"], g["dtable"])
    again = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0, want_dtable=False)
    assert torch.equal(again["dh"], g["dh"])


@pytest.mark.parametrize("rows,vocab,width,cap", [
    (1030, 2500, 65, 0.0), (1500, 777, 128, 30.0), (3001, 1201, 96, 5.0), (8300, 300, 24, 30.0), (1030, 4500, 1001, 0.0), (4111, 1200, 904, 30.0)])
def test_element_by_element(rows, vocab, width, cap):
    """Against the oracle's bounds, in which the target's element of dz is not rounded."""
    h, table, t, targets, up = _problem(rows, vocab, width, rows, True)
    h[::2] += (6.0 * table[targets.clamp(min=0)].float()).to(BF16)[::2]
    nh, nt, nu = _np(h), _np(table), _np(up)
    f = L.cross_entropy(h, table, targets, cap=cap)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=cap)
    want, bound = E.cross_entropy_backward(nh, nt, t, nu, cap), E.cross_entropy_bounds(nh, nt, t, nu, cap, True)
    for n in ("dh", "dtable"):
        worst = np.abs(_np(g[n]) - want[n]) / np.maximum(bound[n], 1e-300)
        assert (worst <= 1.0).all(), (n, float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("rows,vocab,width", [(2048, 3001, 720), (4101, 3001, 360), (9000, 16000, 40), (17000, 1100, 300)])
def test_workspace_stream_and_graph(rows, vocab, width):
    """The sums by sorted targets in just the bytes that the call asks for, over anything; on another stream; and captured,
    replayed between eager calls, with other values in the inputs: the same bits."""
    a, b = (_problem(rows, vocab, width, k, True) for k in (1, 2))
    problems = [(h, table, targets, up) for h, table, _, targets, up in (a, b)]
    need = L.cross_entropy_backward_workspace_bytes(rows, vocab, width, L.MESA_DTYPE_BF16)
    room = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")

    def call(h, table, targets, up, workspace=None):
        f = L.cross_entropy(h, table, targets, cap=30.0)
        return list(L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0, workspace=workspace).values())

    want = [call(*p) for p in problems]
    for k in range(2):
        room[need:] = 0xA5
        assert all(torch.equal(x, y) for x, y in zip(call(*problems[k], workspace=room[:need]), want[k]))
        assert bool((room[need:] == 0xA5).all())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = call(*problems[0])
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    held = [t.clone() for t in problems[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = call(*held, workspace=room[:need])
    for k in range(4):
        for t, s in zip(held, problems[k % 2]):
            t.copy_(s)
        for t in kept:
            t.fill_(3)
        room[:need] = 0xFF
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(kept, want[k % 2])), k
        assert all(torch.equal(x, y) for x, y in zip(call(*problems[1 - k % 2], workspace=room[:need]), want[1 - k % 2])), k


def test_rows_that_do_not_count():
    """NaN in them, in their lse and dloss; and no row that counts at all."""
    rows, vocab, width = 4100, 3001, 360
    h, table, t, targets, up = _problem(rows, vocab, width, 5, True)
    f = L.cross_entropy(h, table, targets, cap=30.0)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0)
    away = targets < 0
    h[away], f["lse"][away], up[away] = float("nan"), float("nan"), float("inf")
    other = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=30.0)
    assert all(torch.equal(g[n], other[n]) for n in g) and bool((g["dh"][away] == 0).all())
    none = L.cross_entropy_backward(h, table, targets * 0 - 1, f["lse"], up, cap=30.0)
    assert not bool(none["dh"].any()) and not bool(none["dtable"].any())
