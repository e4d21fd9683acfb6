"""The example that trains a Hawk layer and a Mesa layer together from 8-bit checkpoints."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_hawk_mesa
    return train_hawk_mesa


def test_example_learns_and_decodes():
    """The loss of guessing is ln 32 = 3.47; the block has to get well below it, and tokens decoded
    one at a time have the whole sequence's logits (fp32, eight CG steps on both sides)."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ex = _example()
    block, losses = ex.train(60, say=lambda m: print(m, flush=True))
    assert np.all(np.isfinite(losses)) and losses[-1] < 0.6 * losses[0]
    assert ex.check_decode(block, say=lambda m: print(m, flush=True)) <= 1e-3


def test_example_gradients_against_differences():
    """Every weight's gradient along a random direction against a central difference of the loss.
    Quantising the activations moves a gradient by about 2^-8 of its terms; a few terms of one
    direction may nearly cancel, hence a bound in parts of the gradient's own length."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ex = _example()
    block = ex.Block("cuda")
    tokens, reset, answers = ex.batch(torch.Generator().manual_seed(3), "cuda", rows=2, length=150)
    there = answers >= 0

    def loss():
        logits, _ = block.forward(tokens, reset, keep=False)
        return float(-torch.log_softmax(logits.double(), dim=-1)[there, answers[there]].sum())

    logits, kept = block.forward(tokens, reset)
    d = torch.softmax(logits, dim=-1)
    d[there, answers[there]] -= 1.0
    grads = block.backward(kept, torch.where(there[..., None], d, 0.0))
    assert set(grads) == set(block.p)
    for n, g in grads.items():
        way = g / g.norm()
        old, size = block.p[n], 1e-2 * float(block.p[n].norm()) / max(1.0, float(block.p[n].numel()) ** 0.5)
        size = max(size, 1e-3)
        block.p[n] = old + size * way
        hi = loss()
        block.p[n] = old - size * way
        lo = loss()
        block.p[n] = old
        want, got = (hi - lo) / (2.0 * size), float((g * way).sum())
        print("%-9s along its gradient: %.5f, by differences %.5f" % (n, got, want), flush=True)
        assert abs(got - want) <= 0.03 * abs(want), n
