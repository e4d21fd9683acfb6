"""A language model's two ends called as a program calls them: together, on one tied table; on another stream and in
captured graphs; in one workspace for all calls; at offsets and sizes past 32 bits.

Tolerances as in tests/test_gpu_vocab.py."""
import numpy as np
import pytest

from oracle import language_ends as E
from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
CAP = 20.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _np(t):
    return t.double().cpu().numpy()


def _within(got, want, bound, name):
    worst = np.abs(_np(got) - want) / np.maximum(bound, 1e-300)
    assert (worst <= 1.0).all(), (name, float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))


def _inputs(rows, vocab, width, dtype, seed):
    rng = np.random.default_rng(seed)
    table = torch.from_numpy((rng.standard_normal((vocab, width)) * 0.3).astype(np.float32)).cuda().to(dtype)
    t = np.minimum((np.exp(rng.random(rows + 1) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1)
    tokens, targets = t[:-1].copy(), t[1:].copy()
    targets[rng.random(rows) < 0.1] = -100
    up = (rng.random(rows) / rows).astype(np.float32)
    return table, torch.from_numpy(tokens).cuda(), torch.from_numpy(targets).cuda(), torch.from_numpy(up).cuda()


def _step(table, tokens, targets, up, scale=1.0, workspace=None):
    """A step of a model whose layers are the identity: every result of the two ends, the table's gradient last."""
    h = L.embedding(table, tokens, scale=scale)
    f = L.cross_entropy(h, table, targets, cap=CAP, want_best=True, workspace=workspace)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=CAP, workspace=workspace)
    head = g["dtable"] * 1
    L.embedding_backward(tokens, g["dh"], table.shape[0], scale=scale, out=g["dtable"], accumulate=True, workspace=workspace)
    return [h, f["loss"], f["lse"], f["best"], g["dh"], head, g["dtable"]]


SIZES = [(1, 50, 64), (300, 777, 72), (2500, 1000, 64)]


@pytest.mark.parametrize("rows,vocab,width", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step_on_a_tied_table(rows, vocab, width, dtype):
    """Against the oracle from end to end: a scale of 2 is exact, so the hidden rows are; what the gradient of the
    head may be off by passes through the look-up's, which adds it up and rounds once."""
    table, tokens, targets, up = _inputs(rows, vocab, width, dtype, rows)
    h, loss, lse, _, dh, head, total = _step(table, tokens, targets, up, scale=2.0)
    nt, t, y, u = _np(table), tokens.cpu().numpy(), targets.cpu().numpy(), _np(up)
    nh = E.embedding(nt, t, 2.0)
    assert (_np(h) == nh).all()
    want, g = E.cross_entropy(nh, nt, y, CAP), E.cross_entropy_backward(nh, nt, y, u, CAP)
    bound = E.cross_entropy_bounds(nh, nt, y, u, CAP, dtype is BF16)
    for n, got in (("lse", lse), ("loss", loss)):
        _within(got, want[n], bound[n], n)
    for n, got in (("dh", dh), ("dtable", head)):
        _within(got, g[n], bound[n], n)
    full, size, count = E.embedding_backward(t, g["dh"], vocab, 2.0, g["dtable"])
    moved, _, _ = E.embedding_backward(t, bound["dh"], vocab, 2.0, bound["dtable"])
    most = (count + 3) * 2.0 ** -24 * (size + np.abs(g["dtable"]) + moved) + moved + HALF[dtype] * (np.abs(full) + moved) * 1.001
    _within(total, full, most, "total")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_tied_gradient_against_differences(dtype):
    """The step's whole gradient along directions, against central differences of the oracle's loss, both ends moved.
    With a step of s the third derivative is s^2 / 6 of itself, some 2^-20 here; the gradient's own bound, summed
    along the direction, is the tolerance beside it."""
    table, tokens, targets, up = _inputs(40, 60, 64, dtype, 3)
    total = _np(_step(table, tokens, targets, up, scale=2.0)[-1])
    nt, t, y, u = _np(table), tokens.cpu().numpy(), targets.cpu().numpy(), _np(up)

    def loss(e):
        return float((E.cross_entropy(E.embedding(e, t, 2.0), e, y, CAP)["loss"] * u).sum())

    nh = E.embedding(nt, t, 2.0)
    g, bound = E.cross_entropy_backward(nh, nt, y, u, CAP), E.cross_entropy_bounds(nh, nt, y, u, CAP, dtype is BF16)
    full, size, count = E.embedding_backward(t, g["dh"], 60, 2.0, g["dtable"])
    moved, _, _ = E.embedding_backward(t, bound["dh"], 60, 2.0, bound["dtable"])
    most = (count + 3) * 2.0 ** -24 * (size + np.abs(g["dtable"]) + moved) + moved + HALF[dtype] * (np.abs(full) + moved) * 1.001
    rng = np.random.default_rng(0)
    for _ in range(5):
        way = rng.standard_normal(nt.shape)
        way /= np.linalg.norm(way)
        s = 2.0 ** -9
        slope = (loss(nt + s * way) - loss(nt - s * way)) / (2 * s)
        assert abs(slope - (total * way).sum()) <= (most * np.abs(way)).sum() + 2.0 ** -18 * max(1.0, abs(slope))


@pytest.mark.parametrize("rows,vocab,width", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_other_stream_and_graph(rows, vocab, width, dtype):
    """The same bits on a stream of one's own and from a captured step, replayed between eager ones and with other
    values in its inputs."""
    a, b = _inputs(rows, vocab, width, dtype, 1), _inputs(rows, vocab, width, dtype, 2)
    want, other = _step(*a), _step(*b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = _step(*a)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    held = [t.clone() for t in a]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = _step(*held)
    for k in range(6):
        source, expect = (a, want) if k % 2 == 0 else (b, other)
        for t, s in zip(held, source):
            t.copy_(s)
        for t in kept:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(kept, expect)), k
        again = _step(*b)
        assert all(torch.equal(x, y) for x, y in zip(again, other)), k


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_graphs_in_one_workspace(dtype):
    """Two captured steps of other sizes share a workspace; they are replayed in turn, with eager calls in it between."""
    sizes = [(300, 777, 72), (2500, 1000, 64)]
    code = L.MESA_DTYPE_F32 if dtype is F32 else L.MESA_DTYPE_BF16
    most = max(max(L.embedding_backward_workspace_bytes(*s), L.cross_entropy_workspace_bytes(*s, code),
                   L.cross_entropy_backward_workspace_bytes(*s, code)) for s in sizes)
    workspace = torch.empty(most, dtype=torch.uint8, device="cuda")
    inputs = [_inputs(*s, dtype, 7) for s in sizes]
    want = [_step(*x) for x in inputs]
    graphs, kept = [], []
    for x in inputs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kept.append(_step(*x, workspace=workspace))
    for k in range(6):
        for t in kept[k % 2]:
            t.fill_(3)
        graphs[k % 2].replay()
        eager = _step(*inputs[1 - k % 2], workspace=workspace)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(kept[k % 2], want[k % 2])), k
        assert all(torch.equal(x, y) for x, y in zip(eager, want[1 - k % 2])), k


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_workspace_for_every_call(dtype):
    """Calls of other sizes one after the other in just the bytes that each asks for, over what the last one left (and
    NaN before the first): the results are those of a workspace of their own, and nothing behind the bytes is written."""
    code = L.MESA_DTYPE_F32 if dtype is F32 else L.MESA_DTYPE_BF16
    shapes = [(300, 777, 72), (1, 5003, 64), (2500, 1000, 64), (33, 1, 1), (20000, 70, 8), (64, 300, 200), (700, 90, 30)]
    inputs = [_inputs(*s, dtype, k) for k, s in enumerate(shapes)]
    most = max(max(L.embedding_backward_workspace_bytes(*s), L.cross_entropy_workspace_bytes(*s, code),
                   L.cross_entropy_backward_workspace_bytes(*s, code)) for s in shapes)
    buf = torch.full((most + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    for s, (table, tokens, targets, up) in list(zip(shapes, inputs)) * 2:
        h = L.embedding(table, tokens)
        f = L.cross_entropy(h, table, targets, cap=CAP, want_best=True)
        calls = [(lambda w: L.cross_entropy(h, table, targets, cap=CAP, want_best=True, workspace=w), L.cross_entropy_workspace_bytes(*s, code)),
                 (lambda w: L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=CAP, workspace=w),
                  L.cross_entropy_backward_workspace_bytes(*s, code)),
                 (lambda w: {"y": L.embedding_backward(tokens, h, s[1], workspace=w)}, L.embedding_backward_workspace_bytes(*s))]
        for k, (call, need) in enumerate(calls):
            want = call(None)
            buf[need:] = 0xA5
            got = call(buf[:need])
            assert all(torch.equal(got[n], want[n]) for n in want), (s, k)
            assert bool((buf[need:] == 0xA5).all()), (s, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_does_not_hang_on_its_neighbours(dtype):
    """What a row gets is the same beside near logits, far ones and NaN."""
    table, tokens, targets, up = _inputs(200, 900, 64, dtype, 5)
    targets[targets < 0] = 3
    h = L.embedding(table, tokens)
    f = L.cross_entropy(h, table, targets, cap=CAP, want_best=True)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=CAP, want_dtable=False)
    odd = torch.arange(200, device="cuda") % 3 == 1
    for value in (1000.0, float("nan"), 0.0):
        other = h.clone()
        other[odd] = value
        fo = L.cross_entropy(other, table, targets, cap=CAP, want_best=True)
        go = L.cross_entropy_backward(other, table, targets, fo["lse"], up, cap=CAP, want_dtable=False)
        assert all(torch.equal(fo[n][~odd], f[n][~odd]) for n in f) and torch.equal(go["dh"][~odd], g["dh"][~odd])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_steps_at_once(dtype):
    """Steps of two sizes on two streams, over each other several times: each has the bits that it has alone."""
    inputs = [_inputs(2500, 1000, 64, dtype, 8), _inputs(700, 3001, 200, dtype, 9)]
    want = [_step(*x) for x in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(_step(*inputs[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            assert all(torch.equal(x, y) for x, y in zip(out, want[k]))


@pytest.mark.parametrize("width", [1, 7, 64, 100, 321])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gaps_are_not_read(dtype, width):
    """What lies between spaced rows, behind the last one and before the first may be NaN."""
    table, tokens, targets, up = _inputs(130, 300, width, dtype, 4)
    h = L.embedding(table, tokens)

    def spaced(x):
        room = torch.full((x.shape[0] * (width + 3) + 70,), float("nan"), dtype=dtype, device="cuda")
        rows = room[33:33 + x.shape[0] * (width + 3)].view(x.shape[0], width + 3)[:, :width]
        rows.copy_(x)
        return rows

    a, b = (h, table), (spaced(h), spaced(table))
    f, g = (L.cross_entropy(*x, targets, cap=CAP, want_best=True) for x in (a, b))
    assert all(torch.equal(f[n], g[n]) for n in f)
    f, g = (L.cross_entropy_backward(*x, targets, f["lse"], up, cap=CAP) for x in (a, b))
    assert all(torch.equal(f[n], g[n]) for n in f)
    assert torch.equal(L.embedding(b[1], tokens), h)
    assert torch.equal(L.embedding_backward(tokens, b[0], 300), L.embedding_backward(tokens, h, 300))


# ------------------------------------------------------------------ far offsets
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_past_32_bits(dtype):
    """A table, hidden rows and gradients whose rows lie 32768 apart, 70000 of them: the last start past 2^31 elements."""
    vocab, width, pitch, rows = 70000, 64, 32768, 260
    code = L.MESA_DTYPE_F32 if dtype is F32 else L.MESA_DTYPE_BF16
    table, tokens, targets, up = _inputs(rows, vocab, width, dtype, 6)
    tokens[:4] = torch.tensor([vocab - 1, vocab - 2, vocab - 1, vocab], device="cuda")
    targets[:2] = torch.tensor([vocab - 1, vocab - 1], device="cuda")
    big = torch.empty((vocab, pitch), dtype=dtype, device="cuda")
    far, far_grad, far_loss = big[:, :width], big[:, 128:128 + width], big[:, 256:256 + width]
    far.copy_(table)
    h = L.embedding(table, tokens)
    assert torch.equal(L.embedding(far, tokens), h)
    f = L.cross_entropy(h, table, targets, cap=CAP, want_best=True)
    ff = L.cross_entropy(h, far, targets, cap=CAP, want_best=True)
    assert all(torch.equal(f[n], ff[n]) for n in f)
    g = L.cross_entropy_backward(h, table, targets, f["lse"], up, cap=CAP)
    far_grad.fill_(7.0)
    want = L.embedding_backward(tokens, h, vocab)
    L.embedding_backward(tokens, h, vocab, out=far_grad)
    assert torch.equal(far_grad, want)
    # the binding hands out dense gradients, the C entry point takes a pitch
    lib, dh = L.load(), torch.empty_like(h)
    need = lib.mesa_cross_entropy_backward_workspace_bytes(rows, vocab, width, code)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    st = lib.mesa_cross_entropy_backward(h.data_ptr(), far.data_ptr(), targets.data_ptr(), 8, f["lse"].data_ptr(), up.data_ptr(), CAP, rows,
                                         vocab, width, width, pitch, code, width, pitch, dh.data_ptr(), far_loss.data_ptr(), ws.data_ptr(),
                                         need, torch.cuda.current_stream().cuda_stream)
    assert st == L.MESA_OK and torch.equal(dh, g["dh"]) and torch.equal(far_loss, g["dtable"])
    # hidden rows far apart: as many as the table has
    many = torch.arange(vocab, device="cuda", dtype=torch.int32) % 50
    few = table[:50].contiguous()
    a, b = L.cross_entropy(table, few, many, cap=CAP), L.cross_entropy(far, few, many, cap=CAP)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_most_rows():
    """2^24 tokens: of whole numbers every sum is exact.  First spread over a table, then all the same."""
    rows, vocab, width = 1 << 24, 1000, 8
    gen = torch.Generator(device="cuda").manual_seed(0)
    tokens = torch.randint(-3, vocab + 3, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    dy = torch.randint(-2, 3, (rows, width), generator=gen, device="cuda").to(BF16)
    got = L.embedding_backward(tokens, dy, vocab, grad_dtype=F32)
    there = (tokens >= 0) & (tokens < vocab)
    want = torch.zeros((vocab, width), device="cuda", dtype=torch.float64)
    want.index_add_(0, tokens[there].long(), dy[there].double())
    assert torch.equal(got.double(), want)
    tokens.fill_(999)
    got = L.embedding_backward(tokens, torch.ones_like(dy), vocab, grad_dtype=F32)
    assert bool((got[999] == 2.0 ** 24).all()) and not bool(got[:999].any())
    with pytest.raises(L.MesaError) as e:
        L.embedding_backward(torch.zeros(rows + 1, device="cuda", dtype=torch.int32), torch.zeros((rows + 1, width), device="cuda"), vocab)
    assert e.value.status == L.MESA_ERR_SHAPE


def test_largest_table():
    """As many rows of one channel as a table may have, 2^31 - 1025 of them: the last is found, and all others are 0."""
    vocab = (1 << 31) - 1025
    table = torch.zeros((vocab, 1), dtype=BF16, device="cuda")
    table[-1] = 3.0
    tokens = torch.tensor([vocab - 1, 0, vocab, -1], device="cuda")
    y = L.embedding(table, tokens)
    assert y.flatten().tolist() == [3.0, 0.0, 0.0, 0.0]
    f = L.cross_entropy(y[:1], table, tokens[:1], want_best=True)
    # exp(9) and 2^31 - 1026 times 1: tiles of equal sums, whose sums are whole numbers
    want = np.log(float(vocab - 1) + np.exp(9.0))
    assert int(f["best"]) == vocab - 1 and abs(float(f["lse"]) - want) < 1e-4 and abs(float(f["loss"]) - (want - 9.0)) < 1e-4
    table.fill_(7.0)
    L.embedding_backward(tokens, torch.ones((4, 1), dtype=BF16, device="cuda"), vocab, out=table)
    assert float(table[0]) == 1.0 and float(table[-1]) == 1.0 and int(torch.count_nonzero(table[1:-1])) == 0
