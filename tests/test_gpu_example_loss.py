"""The trained example's loss and its gradients, against the logits that its forward forms."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_loss_and_gradients():
    """The loss that training takes is the mean of the logits' log-softmax, and every weight's gradient is that of the
    same step by way of the logits.  The head's inputs are fp32 here and 8-bit checkpoints there (2^-8 of their
    group's largest), which moves the gradient of the logits' weights alone; the rest differs by fp32 sums."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_hawk_mesa as ex
    block = ex.Block("cuda")
    tokens, reset, answers = ex.batch(torch.Generator().manual_seed(5), "cuda", rows=3, length=170)
    there = answers >= 0
    logits, kept = block.forward(tokens, reset)
    logp = torch.log_softmax(logits.double(), dim=-1)
    want = -logp[there, answers[there]].mean()
    d = logp.exp()
    d[there, answers[there]] -= 1.0
    way = block.backward(kept, (torch.where(there[..., None], d, 0.0) / there.sum()).float())
    out, kept = block.features(tokens, reset)
    loss, dout, dlogits = block.loss(out, answers)
    assert abs(float(loss) - float(want)) <= 2.0 ** -18 * max(1.0, float(logits.abs().max()))
    got = dict(block.features_backward(kept, dout), logits=dlogits)
    assert set(got) == set(block.p)
    for n in block.p:
        off = float((got[n].double() - way[n].double()).norm() / way[n].double().norm())
        print("%-9s %.1e" % (n, off), flush=True)
        assert off <= (2.0 ** -7 if n == "logits" else 1e-3), n
