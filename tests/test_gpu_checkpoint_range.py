"""Checkpoints over all of fp32, subnormal groups and the largest among them: the kernels' codes, exponents and restored
values are the oracle's, from mesa_checkpoint_pack and from the recurrence's forward."""
import numpy as np
import pytest

from oracle import recurrence as R
from paper_2506_05233_amd import libmesa as L
from test_oracle_checkpoint_bound import TOP, _groups

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lo,hi", [(-149, -120), (-120, 121), (121, 127.999)])
def test_codes_over_all_magnitudes(lo, hi, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x = torch.from_numpy(_groups(np.minimum(np.exp2(np.linspace(lo, hi, 1000)), TOP)).astype(np.float32)).cuda().to(dtype)
    if dtype is torch.bfloat16:
        x = torch.nan_to_num(x.float(), posinf=3.38e38, neginf=-3.38e38).to(dtype)    # rounded up past the largest
    codes, byte, value = R.checkpoint(x.double().cpu().numpy())
    held = L.recurrence(x[None], x[None], x[None], torch.zeros(32, device="cuda"), want_checkpoints=True)
    for ck in [L.checkpoint_pack(x)] + [held[n] for n in ("x", "r", "i")]:
        assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.exponents.cpu().numpy(), byte)
    assert np.array_equal(L.checkpoint_unpack(ck, torch.float32).double().cpu().numpy().reshape(value.shape), value)
    assert np.array_equal(L.checkpoint_unpack(ck).double().cpu().numpy().reshape(value.shape), value)
