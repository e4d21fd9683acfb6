"""The trained example takes tokens, answers and single columns of them as slices of a larger batch."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_slices():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_hawk_mesa as ex
    block = ex.Block("cuda")
    tokens, reset, answers = ex.batch(torch.Generator().manual_seed(6), "cuda", rows=4, length=100)
    reset.zero_()
    part, ends = reset[:, :70].contiguous(), answers[:, :70]
    assert not tokens[:, :70].is_contiguous()
    out, kept = block.features(tokens[:, :70], part)
    loss, dout, dlogits = block.loss(out, ends)
    grads = dict(block.features_backward(kept, dout), logits=dlogits)
    dense, held = block.features(tokens[:, :70].contiguous(), part)
    want, dwant, dl = block.loss(dense, ends.contiguous())
    same = dict(block.features_backward(held, dwant), logits=dl)
    assert torch.equal(out, dense) and torch.equal(loss, want) and all(torch.equal(grads[n], same[n]) for n in same)
    _, state = block.forward(tokens[:, :70], part, keep=False)
    _, other = block.forward(tokens[:, :70].contiguous(), part, keep=False)
    assert torch.equal(block.decode(tokens[:, 70], state), block.decode(tokens[:, 70].contiguous(), other))
