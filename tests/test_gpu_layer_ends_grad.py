"""GPU parity of the gradients of the layer's front end and back end against the fp64 oracle
(oracle/layer_ends.py), through the C ABI.

fp32 results are compared at relative L2 1e-5, as the forward's are (fp32 arithmetic with the
hardware exponential; sums over tokens in fp32); results rounded to bf16 within 2^-8 of an
element plus that error at the array's scale.  From an 8-bit checkpoint the oracle takes the
values that the checkpoint stands for, so the same tolerances hold."""
import numpy as np
import pytest

from mesa_testutil import rel_l2
from oracle import layer_ends as E
from oracle import recurrence as R
from paper_2506_05233_amd import libmesa as L
from paper_2506_05233_amd import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _round(a, dtype):
    a = np.asarray(a, np.float32)
    return W.round_to_bf16(a) if dtype == "bf16" else a


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _close(got, want, dtype, name):
    got = _np(got)
    assert got.shape == want.shape, name
    if dtype == "bf16":
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 4.0 * TOL * np.sqrt(np.mean(want ** 2))), name
    else:
        assert rel_l2(got, want) <= TOL, (name, rel_l2(got, want))


PROJ, FP32 = ("qp", "kp", "vp"), ("conv_q", "conv_k", "conv_v", "a_gamma", "a_beta", "theta")
GRADS = ("dq", "dk", "dv", "dgamma", "dbeta", "dlam")


def _inputs(B, T, H, dk, dv, dtype, seed, conv_v=True):
    rng = np.random.default_rng(seed)
    x = {n: _round(rng.standard_normal((B, T, H, d)), dtype) for n, d in zip(PROJ, (dk, dk, dv))}
    for n, d in zip(FP32[:3], (dk, dk, dv)):
        x[n] = rng.normal(0, 0.5, (H * d, 4)).astype(np.float32)
    x["a_gamma"], x["a_beta"] = (rng.normal(m, 1.5, (B, T, H)).astype(np.float32) for m in (4.0, 0.0))
    x["theta"] = rng.standard_normal((H, dk)).astype(np.float32)
    if not conv_v:
        x["conv_v"] = None
    for n, s in zip(GRADS, ((B, H, T, dk), (B, H, T, dk), (B, H, T, dv), (B, H, T), (B, H, T), (H, dk))):
        x[n] = rng.standard_normal(s).astype(np.float32)
    return x


def _front(x, dtype, kept8, cap=0.9975, eps=1e-6, grad=None):
    grad = dtype if grad is None else grad
    d = {n: None if a is None else torch.from_numpy(a).cuda() for n, a in x.items()}
    held = dict(x)
    for n in PROJ:
        d[n] = d[n].to(_tdt(dtype))
        if kept8:
            B, T, H, w = x[n].shape
            packed = L.checkpoint_pack(d[n].view(B, T, H * w))
            d[n] = L.Checkpoint(packed.buffer, (B, T, H, w))
            held[n] = R.checkpoint(x[n].reshape(B * T, H * w))[2].reshape(x[n].shape)
    got = L.frontend_backward(*(d[n] for n in PROJ + FP32 + GRADS), gamma_cap=cap, l2_eps=eps, grad_dtype=_tdt(grad))
    torch.cuda.synchronize()
    want = E.frontend_backward(**held, gamma_cap=cap, l2_eps=eps)
    assert set(got) == {n for n in want if want[n] is not None}
    for n in got:
        _close(got[n], want[n], grad if n in ("dqp", "dkp", "dvp") else "f32", n)
    return d, got


@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("dtype,kept8", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
def test_frontend_gradients(dk, dv, dtype, kept8):
    """Several runs of a head and a ragged end, values with their filter and without."""
    _front(_inputs(2, 3 * 256 + 11, 3, dk, dv, dtype, dk + dv, conv_v=dk == 64), dtype, kept8)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 15, 16, 17, 33, 128, 131])
def test_frontend_gradients_short(T):
    """Sequences shorter than the filter and around a run of tokens; the cap off; types apart; a
    projection row of zeros."""
    x = _inputs(2, T, 2, 128, 64, "f32", T, conv_v=T % 2 == 1)
    x["kp"][0, 0, 1] = 0.0
    _front(x, "f32", T % 3 == 0, cap=1.0 if T % 4 == 2 else 0.9975, grad="bf16" if T % 5 == 1 else "f32")


def test_frontend_gradients_many_tokens():
    """Enough sequences for long runs of tokens a group of lanes, in bf16 from 8 bits."""
    _front(_inputs(4, 1100, 16, 64, 64, "bf16", 3), "bf16", True)


def test_frontend_gradients_empty():
    x = _inputs(2, 5, 2, 64, 64, "f32", 0)
    d = {n: torch.from_numpy(a).cuda() for n, a in x.items()}
    for n in PROJ + ("a_gamma", "a_beta"):
        d[n] = d[n][:, :0].contiguous()
    for n in GRADS[:5]:
        d[n] = d[n][:, :, :0].contiguous()
    g = L.frontend_backward(*(d[n] for n in PROJ + FP32 + GRADS))
    assert not any(g["dconv_" + n].any() for n in "qkv") and g["dqp"].shape == (2, 0, 2, 64)
    _close(g["dtheta"], E.frontend_backward(**x)["dtheta"], "f32", "dtheta")
    o = torch.zeros((2, 2, 0, 64), device="cuda")
    n = L.output_norm_backward(o, torch.ones((2, 64), device="cuda"), o.view(2, 0, 2, 64))
    assert not n["dweight"].any() and n["do"].shape == o.shape


def test_frontend_gradients_against_differences():
    """The kernels' own loss along random directions: a central difference with a step of 2^-7 of
    the inputs, off by the third derivative times the step squared and the loss's rounding."""
    x = _inputs(2, 70, 2, 64, 64, "f32", 77)
    d = {n: torch.from_numpy(a).cuda() for n, a in x.items()}
    g = L.frontend_backward(*(d[n] for n in PROJ + FP32 + GRADS))

    def loss(e):
        f = L.frontend(*(e[n] for n in PROJ + FP32))
        return sum(float((f[n].double() * d["d" + n].double()).sum()) for n in ("q", "k", "v", "gamma", "beta", "lam"))

    rng = np.random.default_rng(4)
    for n in PROJ + FP32:
        way = torch.from_numpy(rng.standard_normal(x[n].shape).astype(np.float32)).cuda() * 2.0 ** -7
        want = (loss(dict(d, **{n: d[n] + way})) - loss(dict(d, **{n: d[n] - way}))) / 2.0
        got = float((g["d" + n].double() * way.double()).sum())
        size = float(g["d" + n].double().norm() * way.double().norm()) / np.sqrt(way.numel())
        assert abs(got - want) <= 2e-3 * abs(want) + 5e-3 * size, (n, got, want)


@pytest.mark.parametrize("dv", [64, 128])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("kept8", [False, True])
@pytest.mark.parametrize("T", [1, 17, 389])
def test_output_norm_gradients(dv, grad, kept8, T):
    rng = np.random.default_rng(dv + T)
    B, H = 2, 3
    o = (rng.standard_normal((B, H, T, dv)) * rng.uniform(0.01, 10, (B, H, T, 1))).astype(np.float32)
    o[0, 0, 0] = 0.0
    w = rng.normal(1.0, 0.2, (H, dv)).astype(np.float32)
    dy = _round(rng.standard_normal((B, T, H, dv)), grad)
    held, dev_o = o, torch.from_numpy(o).cuda()
    if kept8:
        dev_o = L.checkpoint_pack(dev_o)
        held = R.checkpoint(o.reshape(-1, dv))[2].reshape(o.shape)
    g = L.output_norm_backward(dev_o, torch.from_numpy(w).cuda(), torch.from_numpy(dy).cuda().to(_tdt(grad)), 1e-6)
    torch.cuda.synchronize()
    do, dw = E.output_norm_backward(held, w, dy, 1e-6)
    # a token of zeros has a gradient 1 / sqrt(eps) = 1000 times the others': its own comparison
    got = _np(g["do"])
    zero = np.zeros((B, H, T), bool)
    zero[0, 0, 0] = True
    assert rel_l2(got[zero], do[zero]) <= TOL
    if not zero.all():
        assert rel_l2(got[~zero], do[~zero]) <= TOL
    _close(g["dweight"], dw, "f32", "dweight")


def test_gradients_repeat_bit_for_bit():
    x = _inputs(2, 500, 3, 128, 128, "bf16", 5)
    _, a = _front(x, "bf16", True)
    _, b = _front(x, "bf16", True)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_binding_refuses():
    x = _inputs(1, 4, 1, 64, 64, "f32", 0)
    d = {n: torch.from_numpy(a).cuda() for n, a in x.items()}
    args = [d[n] for n in PROJ + FP32 + GRADS]
    for k, bad, err in ((0, d["qp"].half(), TypeError), (1, L.checkpoint_pack(d["kp"]), TypeError), (3, d["conv_q"][:3], ValueError),
                        (9, d["dq"].bfloat16(), TypeError), (14, d["dlam"].cpu(), ValueError)):
        with pytest.raises(err):
            L.frontend_backward(*args[:k], bad, *args[k + 1:])
    with pytest.raises(L.MesaError) as e:
        L.frontend_backward(*args, gamma_cap=1.5)
    assert e.value.status == L.MESA_ERR_ARG
    with pytest.raises(L.MesaError):
        L.output_norm_backward(d["dq"], d["theta"], d["qp"], eps=float("nan"))
