"""The error that an 8-bit checkpoint makes, over all of fp32 (CPU, on the oracle).

E > -126 is the least that fits, so amax 2^(1 - E) rounds past 127: 2^E / 2 <= amax / 127.5.  E stops at -126, where half a
step is 2^-127; and at 122, where codes stop at 63 since 64 * 2^122 is past fp32."""
import numpy as np
import pytest

from oracle import recurrence as R

TOP = float(np.finfo(np.float32).max)


def _groups(amax, seed=0):
    """Rows of one group each: its largest magnitude, and others below it down to nothing."""
    rng = np.random.default_rng(seed)
    x = rng.uniform(-1.0, 1.0, (len(amax), 32)) * np.asarray(amax)[:, None]
    x[:, 0] = amax
    with np.errstate(under="ignore"):
        return x.astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("lo,hi", [(-149, -120), (-120, -90), (-3, 3), (90, 121), (121, 127.999)])
def test_error_over_all_magnitudes(lo, hi):
    x = _groups(np.minimum(np.exp2(np.linspace(lo, hi, 4001)), TOP))
    codes, byte, value = R.checkpoint(x)
    amax = np.abs(x).max(axis=1)
    step = np.exp2(byte[:, 0] - 127.0)
    clipped = (step == 2.0 ** 122)[:, None] & (np.abs(x) > 63.5 * 2.0 ** 122)
    err = np.abs(value - x)
    assert np.all(err[~clipped] <= np.broadcast_to(step[:, None] / 2, x.shape)[~clipped])
    assert np.all(err[~clipped] <= np.broadcast_to(np.maximum(amax / 127.5, 2.0 ** -127)[:, None], x.shape)[~clipped])
    # what is clipped comes back as 63 2^122, off by less than a step
    assert np.all(np.abs(value[clipped]) == 63 * 2.0 ** 122) and np.all(err[clipped] < 2.0 ** 122)
    assert clipped.any() == (hi > 127)
    # at the least E the error is not within a 127th of the largest magnitude any more
    assert np.any(err > (amax / 127.0)[:, None]) == (lo < -120 or bool(clipped.any()))


def test_the_largest_group_by_hand():
    """127 2^121 still has the codes to 127; from 127.5 2^121 on a group has those to 63 only."""
    x = np.zeros((3, 32))
    x[0, :2] = 127 * 2.0 ** 121, 126.6 * 2.0 ** 121
    x[1, :2] = 127.4 * 2.0 ** 121, 2.0 ** 121
    x[2, :4] = 127.5 * 2.0 ** 121, 63.4 * 2.0 ** 122, 63.6 * 2.0 ** 122, 2.0 ** 121
    codes, byte, value = R.checkpoint(x)
    assert list(byte[:, 0] - 127) == [121, 121, 122]
    assert list(codes[0, :2]) == [127, 127] and list(codes[1, :2]) == [127, 1] and list(codes[2, :4]) == [63, 63, 63, 0]
    assert np.all(value[2, :3] == 63 * 2.0 ** 122)
