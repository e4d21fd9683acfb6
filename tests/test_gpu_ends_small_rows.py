"""Gradients of the layer's ends where a row is so small that its mean square is subnormal and nothing is added to it
(an eps of 0 is allowed).  The forward takes such rows, and the gradient is as finite: n o is of order one.

Rows of 3e-20: a square, 9e-40, is held to 2^-150 / 9e-40 < 8e-7 of itself, so n to half of that and the gradient
to about 1e-6: within the 1e-5 that other rows have.  The front end norms the sum of the squares, not their mean,
so it takes rows of 1e-20 to get there: a square of half of that, 2e-41, is held to 4e-5, the sum of 64 such
independent errors to 4e-5 / sqrt(3 * 64) = 3e-6."""
import numpy as np
import pytest

from oracle import layer_ends as E
from paper_2506_05233_amd import libmesa as L

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


def _close(got, want, name):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), name
    assert np.linalg.norm(got - want) <= TOL * np.linalg.norm(want), name


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1.0, 1e-15, 3e-20])
def test_output_norm_of_small_rows(d, size):
    rng = np.random.default_rng(d)
    B, H, T = 2, 2, 21
    o = (rng.uniform(0.5, 1.0, (B, H, T, d)) * rng.choice([-1.0, 1.0], (B, H, T, d)) * size).astype(np.float32)
    w, dy = rng.normal(1.0, 0.2, (H, d)).astype(np.float32), rng.standard_normal((B, T, H, d)).astype(np.float32)
    t = [torch.from_numpy(a).cuda() for a in (o, w, dy)]
    _close(L.output_norm(t[0], t[1], 0.0, torch.float32), E.output_norm(o, w, 0.0), "y")
    g = L.output_norm_backward(t[0], t[1], t[2], 0.0)
    do, dw = E.output_norm_backward(o, w, dy, 0.0)
    _close(g["do"], do, "do")
    _close(g["dweight"], dw, "dweight")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1.0, 1e-15, 6e-20, 1e-20])
def test_front_end_of_small_rows(d, size):
    """SiLU halves a small value, so the rows that are normed are of half that size."""
    rng = np.random.default_rng(d)
    B, T, H = 1, 21, 2
    p = {n: (rng.uniform(0.7, 1.0, (B, T, H, d)) * rng.choice([-1.0, 1.0], (B, T, H, d)) * size).astype(np.float32) for n in ("qp", "kp", "vp")}
    conv = np.zeros((H * d, 4), np.float32)
    conv[:, 0] = 1.0
    rest = [rng.standard_normal(s).astype(np.float32) for s in ((B, T, H), (B, T, H), (H, d))]
    grads = [rng.standard_normal(s).astype(np.float32) for s in ((B, H, T, d),) * 3 + ((B, H, T),) * 2 + ((H, d),)]
    args = [p["qp"], p["kp"], p["vp"], conv, conv, None] + rest + grads
    g = L.frontend_backward(*(None if a is None else torch.from_numpy(a).cuda() for a in args), l2_eps=0.0)
    want = E.frontend_backward(*args, l2_eps=0.0)
    for n in ("dqp", "dkp", "dconv_q", "dconv_k"):
        _close(g[n], want[n], n)
