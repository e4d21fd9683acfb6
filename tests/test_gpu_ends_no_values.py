"""The front end's gradients where the values passed through unfiltered: their projection is not read, so a
trainer need not keep it."""
import numpy as np
import pytest

from oracle import layer_ends as E
from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.synchronize()


def _inputs(B, T, H, dk, dv, seed):
    rng = np.random.default_rng(seed)
    shapes = dict(qp=(B, T, H, dk), kp=(B, T, H, dk), vp=(B, T, H, dv), conv_q=(H * dk, 4), conv_k=(H * dk, 4), a_gamma=(B, T, H),
                  a_beta=(B, T, H), theta=(H, dk), dq=(B, H, T, dk), dk=(B, H, T, dk), dv=(B, H, T, dv), dgamma=(B, H, T),
                  dbeta=(B, H, T), dlam=(H, dk))
    return {n: rng.standard_normal(s).astype(np.float32) for n, s in shapes.items()}


@pytest.mark.parametrize("T", [1, 37, 300])
@pytest.mark.parametrize("kept8", [False, True])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 64)])
def test_no_projection_of_the_values(T, kept8, dk, dv):
    """The same gradients without vp as with it (bit for bit), and the values' own is dv laid out as they were."""
    x = _inputs(2, T, 3, dk, dv, T + dk)
    d = {n: torch.from_numpy(a).cuda() for n, a in x.items()}
    if kept8:
        for n in ("qp", "kp", "vp"):
            d[n] = L.checkpoint_pack(d[n])
    args = [d[n] for n in ("conv_q", "conv_k")] + [None] + [d[n] for n in ("a_gamma", "a_beta", "theta", "dq", "dk", "dv", "dgamma", "dbeta", "dlam")]
    want = L.frontend_backward(d["qp"], d["kp"], d["vp"], *args, grad_dtype=torch.float32)
    got = L.frontend_backward(d["qp"], d["kp"], None, *args, grad_dtype=torch.float32)
    assert set(got) == set(want) and "dconv_v" not in got
    assert all(torch.equal(got[n], want[n]) for n in want)
    assert torch.equal(got["dvp"], d["dv"].transpose(1, 2).contiguous())
    half = L.frontend_backward(d["qp"], d["kp"], None, *args)["dvp"]
    assert half.dtype == (torch.bfloat16 if kept8 else torch.float32) and torch.equal(half, got["dvp"].to(half.dtype))
    if not kept8:
        ref = E.frontend_backward(x["qp"], x["kp"], x["vp"], x["conv_q"], x["conv_k"], None, *(x[n] for n in (
            "a_gamma", "a_beta", "theta", "dq", "dk", "dv", "dgamma", "dbeta", "dlam")))
        for n in got:
            e = np.linalg.norm(got[n].double().cpu().numpy() - ref[n]) / np.linalg.norm(ref[n])
            assert e <= 1e-5, (n, e)


def test_filtered_values_need_their_projection():
    x = _inputs(1, 5, 1, 64, 64, 0)
    d = {n: torch.from_numpy(a).cuda() for n, a in x.items()}
    rest = [d[n] for n in ("a_gamma", "a_beta", "theta", "dq", "dk", "dv", "dgamma", "dbeta", "dlam")]
    with pytest.raises((TypeError, ValueError)):
        L.frontend_backward(d["qp"], d["kp"], None, d["conv_q"], d["conv_k"], d["conv_q"], *rest)
    with pytest.raises(ValueError):
        L.frontend_backward(d["qp"], d["kp"], None, d["conv_q"], d["conv_k"], None, *rest[:5], rest[5][..., :32], *rest[6:])
