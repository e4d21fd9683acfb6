"""GPU parity of the gated recurrence, its step, its gradients and the 8-bit checkpoints
against the fp64 oracle (oracle/recurrence.py), through the C ABI.

Tolerances.  A kernel's a_t is off by a few units of 2^-24 (the hardware exponential and the
rounding of its argument), and the state at t gathers those of the last N = 1 / (1 - a) tokens;
as independent errors they add to about 4 * 2^-24 * sqrt(N / 2) of the state, below 1e-5 for the
slowest channel here (N about 2000).  A gradient passes through two such walks: 2e-5.  Both are
relative L2 over an array.  An output rounded to bf16 is within 2^-9 of its fp32 value, so within
2^-8 of the oracle's plus the fp32 error at the array's scale, element by element.  The codes and
exponents of a checkpoint are exact."""
import numpy as np
import pytest

from mesa_testutil import rel_l2
from oracle import recurrence as R
from paper_2506_05233_amd import libmesa as L
from paper_2506_05233_amd import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL_STATE, TOL_GRAD = 1e-5, 2e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _say(msg):
    print(msg, flush=True)


def _tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _round(a, dtype):
    a = np.asarray(a, np.float32)
    return W.round_to_bf16(a) if dtype == "bf16" else a


def _inputs(B, T, Wd, dtype, seed, resets=0.0, h0=True):
    """Decays from fast to slow (a open gate keeps 0.5 to 0.999 of the state a token)."""
    rng = np.random.default_rng(seed)
    x = {n: _round(rng.standard_normal((B, T, Wd)), dtype) for n in "xri"}
    keep = np.exp(-np.exp(rng.uniform(np.log(1e-3), np.log(0.7), Wd)))
    x["theta"] = np.log(np.expm1(-np.log(keep) / 8.0)).astype(np.float32)
    x["reset"] = (rng.random((B, T)) < resets).astype(np.uint8) if resets else None
    x["h0"] = rng.standard_normal((B, Wd)).astype(np.float32) if h0 else None
    x["dy"] = _round(rng.standard_normal((B, T, Wd)), dtype)
    x["dfinal"] = rng.standard_normal((B, Wd)).astype(np.float32)
    return x


def _dev(x, dtype):
    return {n: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to(_tdt(dtype) if n in ("x", "r", "i", "dy") else
                                                                   torch.uint8 if n == "reset" else torch.float32)
            for n, a in x.items()}


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _close(got, want, dtype, tol, name):
    got, want = _np(got), np.asarray(want, np.float64)
    assert got.shape == want.shape, name
    if want.size == 0:
        return 0.0
    assert np.all(np.isfinite(got) == np.isfinite(want)), name
    if dtype == "bf16":
        scale = np.sqrt(np.mean(want ** 2))
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 4.0 * tol * scale), name
        return rel_l2(got, want)
    e = rel_l2(got, want)
    assert e <= tol, (name, e)
    return e


def _run(d, **kw):
    return L.recurrence(d["x"], d["r"], d["i"], d["theta"], reset=d["reset"], h0=d["h0"], **kw)


def _check_forward(x, dtype):
    d = _dev(x, dtype)
    f = _run(d, want_final=True, want_states=True, want_checkpoints=True)
    torch.cuda.synchronize()
    ref = R.forward(x["x"], x["r"], x["i"], x["theta"], reset=x["reset"], h0=x["h0"])
    e = [_close(f["y"], ref["y"], dtype, TOL_STATE, "y"), _close(f["h"], ref["h"], "f32", TOL_STATE, "h"),
         _close(f["states"], ref["states"], "f32", TOL_STATE, "states")]
    for n in "xri":
        if x[n].size:
            codes, byte, _ = R.checkpoint(x[n].reshape(-1, x[n].shape[-1]))
            assert np.array_equal(f[n].codes.cpu().numpy(), codes) and np.array_equal(f[n].exponents.cpu().numpy(), byte), n
    return d, f, ref, max(e)


def _check_backward(x, d, f, ref, dtype, kept8, dfinal=True):
    held = {n: (R.checkpoint(x[n].reshape(-1, x[n].shape[-1]))[2].reshape(x[n].shape) if kept8 and x[n].size else x[n]) for n in "xri"}
    states = torch.from_numpy(ref["states"].astype(np.float32)).cuda()
    df = d["dfinal"] if dfinal else None
    src = [f[n] for n in "xri"] if kept8 else [d[n] for n in "xri"]
    g = L.recurrence_backward(*src, d["theta"], states, d["dy"], df, reset=d["reset"])
    torch.cuda.synchronize()
    want = R.backward(held["x"], held["r"], held["i"], x["theta"], ref["states"].astype(np.float32), x["dy"],
                      x["dfinal"] if dfinal else None, reset=x["reset"])
    e = 0.0
    for n in ("dx", "dr", "di"):
        e = max(e, _close(g[n], want[n], dtype, TOL_GRAD, n))
    for n in ("dtheta", "dh0"):
        # where resets cut every sequence from its start dh0 is exactly zero
        if not np.any(want[n]):
            assert not np.any(_np(g[n])), n
        else:
            e = max(e, _close(g[n], want[n], "f32", TOL_GRAD, n))
    return e


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 127, 128, 129, 255, 256, 257, 600, 2049])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths(T, dtype):
    """Lengths around a lane's run, a block and a tile; gradients from the tensors and from 8 bits."""
    x = _inputs(2, T, 72, dtype, seed=T, resets=0.02 if T % 2 else 0.0, h0=T % 3 != 0)
    d, f, ref, e = _check_forward(x, dtype)
    e2 = [_check_backward(x, d, f, ref, dtype, kept8, dfinal=kept8) for kept8 in (False, True)]
    _say("T=%d %s: forward %.1e, gradients %.1e, from 8 bits %.1e" % (T, dtype, e, e2[0], e2[1]))


@pytest.mark.parametrize("width", [1, 3, 4, 31, 32, 63, 64, 65, 130, 320])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_widths(width, dtype):
    """Widths around a lane's four channels, a group of 32 and a slab of 64."""
    x = _inputs(3, 300, width, dtype, seed=1000 + width, resets=0.01 if width % 2 else 0.0)
    d, f, ref, e = _check_forward(x, dtype)
    e2 = [_check_backward(x, d, f, ref, dtype, kept8) for kept8 in (False, True)]
    _say("width %d %s: forward %.1e, gradients %.1e, from 8 bits %.1e" % (width, dtype, e, e2[0], e2[1]))


@pytest.mark.parametrize("T,width,resets", [(129, 64, 0.0), (300, 65, 0.01), (520, 72, 0.0), (257, 130, 0.02), (600, 36, 0.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences(T, width, resets, dtype):
    """Enough sequences to fill the GPU with workgroups of 64 channels (fewer take half of them)."""
    x = _inputs(140, T, width, dtype, seed=T + width, resets=resets)
    d, f, ref, e = _check_forward(x, dtype)
    e2 = [_check_backward(x, d, f, ref, dtype, kept8) for kept8 in (False, True)]
    _say("140 sequences T=%d width %d %s: forward %.1e, gradients %.1e, from 8 bits %.1e" % (T, width, dtype, e, e2[0], e2[1]))


@pytest.mark.parametrize("B", [2, 140])
@pytest.mark.parametrize("dtype,kept8,grad", [("f32", False, "bf16"), ("bf16", False, "f32"), ("f32", True, "f32"), ("bf16", True, "f32"),
                                              ("f32", True, "bf16")])
def test_gradients_of_another_type(B, dtype, kept8, grad):
    """Gradients in fp32 of bf16 or 8-bit inputs and the other way."""
    x = _inputs(B, 270, 68, dtype, seed=B, resets=0.01)
    x["dy"] = _round(x["dy"], "bf16")
    d, f, ref, _ = _check_forward(x, dtype)
    d["dy"] = d["dy"].to(_tdt(grad))
    held = {n: (R.checkpoint(x[n].reshape(-1, 68))[2].reshape(x[n].shape) if kept8 else x[n]) for n in "xri"}
    g = L.recurrence_backward(*((f if kept8 else d)[n] for n in "xri"), d["theta"], f["states"], d["dy"], d["dfinal"], reset=d["reset"])
    want = R.backward(held["x"], held["r"], held["i"], x["theta"], _np(f["states"]), x["dy"], x["dfinal"], reset=x["reset"])
    for n in ("dx", "dr", "di"):
        assert g[n].dtype == _tdt(grad)
        _close(g[n], want[n], grad, TOL_GRAD, n)
    for n in ("dtheta", "dh0"):
        _close(g[n], want[n], "f32", TOL_GRAD, n)


def test_many_tiles():
    """One long sequence: every tile's entering state comes from all those before it."""
    x = _inputs(1, 20011, 8, "f32", seed=5, resets=0.0005)
    d, f, ref, e = _check_forward(x, "f32")
    _say("T=20011: forward %.1e, gradients %.1e" % (e, _check_backward(x, d, f, ref, "f32", False)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 300, 700])
def test_every_token_resets(T, dtype):
    """Rows that keep nothing: each state is its own token's input alone."""
    x = _inputs(2, T, 40, dtype, seed=T, h0=True)
    x["reset"] = np.full((2, T), 255, np.uint8)
    x["h0"][:] = np.nan
    x["r"][:] = np.nan
    d, f, ref, _ = _check_forward_no_kept(x, dtype)
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], f["states"], d["dy"], d["dfinal"], reset=d["reset"])
    assert not np.any(_np(g["dr"])) and not np.any(_np(g["dtheta"])) and not np.any(_np(g["dh0"]))
    si = 1.0 / (1.0 + np.exp(-x["i"].astype(np.float64)))
    dy = x["dy"].astype(np.float64)
    dy[:, -1] += x["dfinal"]
    _close(g["dx"], dy * si, dtype, TOL_GRAD, "dx")


def _check_forward_no_kept(x, dtype):
    """Inputs that may hold NaN and infinities: the same places finite, and those compared."""
    d = _dev(x, dtype)
    f = _run(d, want_final=True, want_states=True)
    ref = R.forward(x["x"], x["r"], x["i"], x["theta"], reset=x["reset"], h0=x["h0"])
    ok = np.isfinite(ref["y"])
    assert np.array_equal(np.isfinite(_np(f["y"])), ok)
    y = torch.where(torch.from_numpy(ok).cuda(), f["y"].float(), 0.0)
    _close(y, np.where(ok, ref["y"], 0.0), dtype, TOL_STATE, "y")
    _close(f["h"], ref["h"], "f32", TOL_STATE, "h")
    return d, f, ref, 0.0


@pytest.mark.parametrize("at", [3, 127, 128, 255, 256, 511, 512, 600])
def test_a_reset_reads_nothing_before_it(at):
    """NaN and infinities before a reset, and in the reset token's own gate, stay there; without
    the reset they reach every later token."""
    x = _inputs(2, 700, 68, "f32", seed=at)
    x["x"][0, at - 2, 5] = np.inf
    x["x"][0, at - 1, 6] = np.nan
    x["r"][0, at, 7] = np.nan
    x["h0"][0, 8] = -np.inf
    bad = _dev(x, "f32")
    y = _run(bad)
    assert not torch.isfinite(y[0, at - 1:, 5:7]).any() and not torch.isfinite(y[0, :, 8]).any()
    assert torch.isnan(y[0, at:, 6]).all() and torch.isnan(y[0, at:, 7]).all() and torch.isfinite(y[1]).all()
    x["reset"] = np.zeros((2, 700), np.uint8)
    x["reset"][0, at] = 1
    d, f, ref, _ = _check_forward_no_kept(x, "f32")
    assert torch.isfinite(f["y"][0, at:]).all()
    dy = d["dy"].clone()
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], f["states"], dy, d["dfinal"], reset=d["reset"])
    x2 = {n: (None if a is None else a.copy()) for n, a in x.items()}
    want = R.backward(x2["x"], x2["r"], x2["i"], x2["theta"], _np(f["states"]), x2["dy"], x2["dfinal"], reset=x2["reset"])
    for n in ("dx", "dr", "di"):
        got = _np(g[n])
        assert np.all(np.isfinite(got[0, at:])) and rel_l2(got[0, at:], want[n][0, at:]) <= TOL_GRAD, n
        assert np.all(np.isfinite(got[1])) and np.all(np.isfinite(got[0]) == np.isfinite(want[n][0])), n


@pytest.mark.parametrize("at,bad", [(2, 3), (5, 6), (130, 131), (130, 170), (300, 699)])
def test_a_reset_hands_no_gradient_back(at, bad):
    """NaN gates and gradients at tokens after a reset do not reach those before it."""
    x = _inputs(2, 700, 68, "f32", seed=bad)
    x["reset"] = np.zeros((2, 700), np.uint8)
    x["reset"][0, at] = 1
    x["r"][0, bad, 7] = np.nan
    x["dy"][0, bad, 9] = np.inf
    x["dfinal"][0, 11] = np.nan
    d = _dev(x, "f32")
    f = L.recurrence(d["x"], d["r"], d["i"], d["theta"], reset=d["reset"], h0=d["h0"], want_states=True)
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], f["states"], d["dy"], d["dfinal"], reset=d["reset"])
    want = R.backward(x["x"], x["r"], x["i"], x["theta"], _np(f["states"]), x["dy"], x["dfinal"], reset=x["reset"])
    assert np.all(np.isfinite(_np(g["dh0"])))
    for n in ("dx", "dr", "di"):
        got = _np(g[n])
        assert not np.isfinite(got[0, bad, 9]) or n == "dr", n
        assert np.all(np.isfinite(got[0, :at])) and np.all(np.isfinite(got[1])), n
        assert rel_l2(got[0, :at], want[n][0, :at]) <= TOL_GRAD and rel_l2(got[1], want[n][1]) <= TOL_GRAD, n


def test_gates_at_their_ends():
    """Gates shut and open past fp32's exponential, no decay at all, a decay that forgets at once."""
    x = _inputs(1, 140, 12, "f32", seed=9)
    x["r"][0, :, 0:4] = np.array([-200.0, -80.0, 80.0, 200.0], np.float32)
    x["i"][0, :, 4:8] = np.array([-200.0, -80.0, 80.0, 200.0], np.float32)
    x["theta"][8:12] = [-120.0, -60.0, 60.0, 300.0]
    d, f, ref, e = _check_forward_no_kept(x, "f32")
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], f["states"], d["dy"], d["dfinal"])
    want = R.backward(x["x"], x["r"], x["i"], x["theta"], _np(f["states"]), x["dy"], x["dfinal"])
    for n in ("dx", "dr", "di", "dtheta", "dh0"):
        got, ref_n = _np(g[n]), want[n]
        assert np.all(np.isfinite(got)), n
        # columns one by one: their scales are far apart.  Where m^2 is below 2^-126 it counts as 0, so an
        # element may be off by 2^-63 |g|, with |g| up to the sum of 140 tokens' dy: below 1e-16 in all
        # (dtheta is one sum a column, so its error goes by the size of its terms, which nearly cancel in some)
        for c in range(12):
            size = want["dtheta_size"][c] if n == "dtheta" else np.linalg.norm(ref_n[..., c])
            assert np.linalg.norm(got[..., c] - ref_n[..., c]) <= TOL_GRAD * size + 1e-16, (n, c)


def test_slices_of_one_projection_and_odd_addresses():
    """x, r, i as slices of one array, dx, dr, di too; and arrays that start off their vector's
    alignment: the same results as from dense ones."""
    for dtype in ("f32", "bf16"):
        x = _inputs(2, 333, 96, dtype, seed=12, resets=0.01)
        d = _dev(x, dtype)
        want = _run(d, want_states=True)
        wg = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], want["states"], d["dy"], d["dfinal"], reset=d["reset"])
        for lead in (0, 1):
            flat = torch.zeros(2 * 333 * 3 * 96 + lead, dtype=_tdt(dtype), device="cuda")
            fused = flat[lead:].view(2, 333, 288)
            fused.copy_(torch.cat([d["x"], d["r"], d["i"]], dim=-1))
            s = dict(d, **dict(zip("xri", fused.split(96, dim=-1))))
            got = _run(s, want_states=True)
            assert torch.equal(got["y"], want["y"]) and torch.equal(got["states"], want["states"])
            grads = torch.empty(2 * 333 * 3 * 96 + lead, dtype=_tdt(dtype), device="cuda")[lead:].view(2, 333, 288)
            g = L.recurrence_backward(s["x"], s["r"], s["i"], d["theta"], want["states"], d["dy"], d["dfinal"], reset=d["reset"],
                                      out=grads.split(96, dim=-1))
            for n in wg:
                assert torch.equal(g[n], wg[n]), (n, lead)
            ck = L.checkpoint_pack(s["r"])
            assert torch.equal(ck.codes, L.checkpoint_pack(d["r"]).codes) and torch.equal(ck.exponents, L.checkpoint_pack(d["r"]).exponents)


def test_a_sequence_in_parts_and_token_by_token():
    """The state handed from one call to the next, and decoding a token at a time."""
    x = _inputs(3, 523, 70, "f32", seed=20, resets=0.01)
    d = _dev(x, "f32")
    whole = _run(d, want_final=True)
    h, parts = d["h0"], []
    for lo, hi in ((0, 0), (0, 1), (1, 257), (257, 520)):
        p = {n: d[n][:, lo:hi].contiguous() for n in ("x", "r", "i", "reset")}
        f = L.recurrence(p["x"], p["r"], p["i"], d["theta"], reset=p["reset"], h0=h, want_final=True)
        parts.append(f["y"])
        h = f["h"]
    for t in range(520, 523):
        old = h.clone()
        new = torch.empty_like(h)
        tok = [d[n][:, t] for n in "xri"]
        y = L.recurrence_step(h, *tok, d["theta"], reset=d["reset"][:, t].contiguous(), state_out=new)
        assert torch.equal(h, old)
        y2 = L.recurrence_step(h, *tok, d["theta"], reset=d["reset"][:, t].contiguous())
        assert torch.equal(h, new) and torch.equal(y, y2)
        parts.append(y[:, None])
    assert rel_l2(_np(torch.cat(parts, dim=1)), _np(whole["y"])) <= TOL_STATE and rel_l2(_np(h), _np(whole["h"])) <= TOL_STATE


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,width", [(1, 1), (1, 2048), (5, 67), (256, 96)])
def test_step(B, width, dtype):
    x = _inputs(B, 1, width, dtype, seed=B + width, resets=0.3)
    d = _dev(x, dtype)
    state = d["h0"].clone()
    y = L.recurrence_step(state, *(d[n][:, 0] for n in "xri"), d["theta"], reset=d["reset"][:, 0].contiguous())
    ref = R.forward(x["x"], x["r"], x["i"], x["theta"], reset=x["reset"], h0=x["h0"])
    _close(state, ref["h"], "f32", TOL_STATE, "state")
    _close(y, ref["y"][:, 0], dtype, TOL_STATE, "y")


def test_empty_and_single():
    dev = "cuda"
    for B, T, Wd in ((0, 5, 8), (2, 0, 8), (2, 5, 0)):
        z = torch.zeros((B, T, Wd), device=dev)
        th, h0 = torch.zeros(Wd, device=dev), torch.ones((B, Wd), device=dev)
        f = L.recurrence(z, z, z, th, h0=h0, want_final=True, want_states=True)
        assert f["y"].shape == (B, T, Wd) and (T > 0 or torch.equal(f["h"], h0))
        g = L.recurrence_backward(z, z, z, th, f["states"], z, h0)
        assert (T > 0 or torch.equal(g["dh0"], h0)) and not g["dtheta"].any()
    assert L.checkpoint_unpack(L.checkpoint_pack(torch.zeros((0, 7), device=dev))).shape == (0, 7)


def test_gradients_against_differences():
    """The kernels' own loss, one direction at a time: a central difference in fp32 with a step of
    2^-6 of the input is off by the third derivative times the step squared (about 1e-4) and by
    the loss's rounding over the step (1e-7 * 64)."""
    x = _inputs(2, 300, 16, "f32", seed=31, resets=0.01)
    d = _dev(x, "f32")
    rng = np.random.default_rng(1)
    f = _run(d, want_states=True)
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], f["states"], d["dy"], d["dfinal"], reset=d["reset"])

    def loss(e):
        f = _run(e, want_final=True)
        return float((f["y"].double() * d["dy"].double()).sum() + (f["h"].double() * d["dfinal"].double()).sum())

    for n in ("x", "r", "i", "theta", "h0"):
        way = torch.from_numpy(rng.standard_normal(d[n].shape).astype(np.float32)).cuda() * 2.0 ** -6
        want = (loss(dict(d, **{n: d[n] + way})) - loss(dict(d, **{n: d[n] - way}))) / 2.0
        got = float((g["d" + n].double() * way.double()).sum())
        size = float(g["d" + n].double().norm() * way.double().norm()) / np.sqrt(way.numel())
        _say("d%s along a direction: %.6f, by differences %.6f" % (n, got, want))
        assert abs(got - want) <= 2e-3 * abs(want) + 2e-3 * size, n


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    """Sums in a fixed order: the same bits from call to call, on a stream of its own, and from
    each replay of a captured graph, with other work between the replays."""
    x = _inputs(2, 1500, 200, "bf16", seed=40, resets=0.002)
    d = _dev(x, "bf16")

    def work():
        f = _run(d, want_final=True, want_states=True, want_checkpoints=True)
        g = L.recurrence_backward(f["x"], f["r"], f["i"], d["theta"], f["states"], d["dy"], d["dfinal"], reset=d["reset"])
        return [f["y"], f["h"], f["states"]] + [f[n].buffer[:2 * 1500 * 200] for n in "xri"] + [g[n] for n in sorted(g)]

    want = work()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = work()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = work()
    for k in range(4):
        for t in kept:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)), k
        again = work()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), k


def test_offsets_past_32_bits():
    """Rows 32768 apart over 70,000 tokens: the last elements lie past 2^31 of the array."""
    T, Wd, pitch = 70000, 64, 32768
    big = torch.empty((1, T, pitch), dtype=torch.bfloat16, device="cuda")
    d = _dev(_inputs(1, T, Wd, "bf16", seed=50, resets=0.001), "bf16")
    for k, n in enumerate("xri"):
        big[:, :, pitch - (k + 1) * Wd:pitch - k * Wd] = d[n]
    far = dict(d, **{n: big[:, :, pitch - (k + 1) * Wd:pitch - k * Wd] for k, n in enumerate("xri")})
    a, b = _run(far, want_final=True, want_states=True), _run(d, want_final=True, want_states=True)
    assert all(torch.equal(a[n], b[n]) for n in a)
    g = L.recurrence_backward(d["x"], d["r"], d["i"], d["theta"], b["states"], d["dy"], d["dfinal"], reset=d["reset"])
    q = L.recurrence_backward(far["x"], far["r"], far["i"], d["theta"], b["states"], d["dy"], d["dfinal"], reset=d["reset"],
                              out=[big[:, :, k * Wd:(k + 1) * Wd] for k in range(3)])
    assert all(torch.equal(q[n], g[n]) for n in g)
    ck = L.checkpoint_pack(far["r"])
    assert torch.equal(ck.codes, L.checkpoint_pack(d["r"]).codes)
    L.checkpoint_unpack(ck, out=far["x"])
    assert torch.equal(far["x"], L.checkpoint_unpack(ck))


# ---------------------------------------------------------------- checkpoints
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width,pad", [(1, 1, 0), (3, 31, 0), (5, 32, 0), (7, 33, 3), (40, 100, 0), (9, 128, 64), (1, 4100, 0), (130, 64, 0)])
def test_checkpoint(rows, width, pad, dtype):
    """Codes, exponents and restored values, exact; magnitudes from 2^-140 to 2^127."""
    rng = np.random.default_rng(rows * 1000 + width)
    x = rng.standard_normal((rows, width)) * np.exp2(rng.integers(-140, 126, (rows, 1)))
    x[0, 0] = 0.0
    if rows > 2:
        x[1] = 0.0
        x[2, 0] = np.inf
        x[2, -1] = np.nan
    if rows > 4:
        x[3, 0] = 3.4e38
        x[4, :5] = [127.5, 127.4375, -127.5, 0.5, 1.5]
        x[4, 5:] = 0.25
    with np.errstate(over="ignore"):
        x = torch.from_numpy(x.astype(np.float32)).to(_tdt(dtype)).float().numpy()
    wide = torch.zeros((rows, width + pad), dtype=_tdt(dtype), device="cuda")
    wide[:, :width] = torch.from_numpy(x).cuda().to(_tdt(dtype))
    ck = L.checkpoint_pack(wide[:, :width])
    codes, byte, value = R.checkpoint(x)
    assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.exponents.cpu().numpy(), byte)
    for out in (torch.float32, torch.bfloat16):
        got = _np(L.checkpoint_unpack(ck, out))
        assert np.array_equal(got, value, equal_nan=True), out
    back = torch.full((rows, width + pad), 7.0, dtype=_tdt(dtype), device="cuda")
    L.checkpoint_unpack(ck, out=back[:, :width])
    assert np.array_equal(_np(back[:, :width]), value, equal_nan=True) and bool((back[:, width:] == 7.0).all())


def test_checkpoint_odd_addresses():
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.randn(64 * 64 + 1, device="cuda").to(dtype)
        x = flat[1:].view(64, 64)
        a, b = L.checkpoint_pack(x), L.checkpoint_pack(x.clone())
        assert torch.equal(a.buffer[:64 * 66], b.buffer[:64 * 66])
        out = torch.empty_like(flat)[1:].view(64, 64)
        assert torch.equal(L.checkpoint_unpack(a, out=out), L.checkpoint_unpack(b, dtype))


# ---------------------------------------------------------------- refusals of the binding
def test_binding_refuses():
    x = torch.zeros((2, 4, 8), device="cuda")
    th = torch.zeros(8, device="cuda")
    st = torch.zeros((2, 1, 8), device="cuda")
    with pytest.raises(TypeError):
        L.recurrence(x.half(), x.half(), x.half(), th)
    with pytest.raises(ValueError):
        L.recurrence(x, x[:, :3], x, th)
    with pytest.raises(ValueError):
        L.recurrence(x, torch.zeros((2, 4, 16), device="cuda")[..., :8], x, th)   # spaced otherwise
    with pytest.raises(ValueError):
        L.recurrence(x.transpose(0, 1), x.transpose(0, 1), x.transpose(0, 1), th)
    with pytest.raises(ValueError):
        L.recurrence(x, x, x, th[:4])
    with pytest.raises(TypeError):
        L.recurrence(x, x, x, th, reset=torch.zeros((2, 4), device="cuda"))
    with pytest.raises(L.MesaError) as e:
        L.recurrence(x, x, x, th, decay=0.0)
    assert e.value.status == L.MESA_ERR_ARG
    with pytest.raises(L.MesaError) as e:
        L.recurrence(x, x, x, th, out=x)
    assert e.value.status == L.MESA_ERR_ARG
    with pytest.raises(TypeError):
        L.recurrence_backward(L.checkpoint_pack(x), x, x, th, st, x)
    with pytest.raises(ValueError):
        L.recurrence_backward(x, x, x, th, st[:, :, :4], x)
    with pytest.raises(ValueError):
        L.checkpoint_pack(x.expand(3, 2, 4, 8))
    with pytest.raises(ValueError):
        L.checkpoint_pack(x.cpu())
    with pytest.raises(ValueError):
        L.Checkpoint(torch.zeros(10, dtype=torch.uint8, device="cuda"), (2, 8))
    with pytest.raises(ValueError):
        L.recurrence_step(st[:, 0], x[:, 0], x[:, 0], x[:, 0], th, state_out=st[:1, 0])
