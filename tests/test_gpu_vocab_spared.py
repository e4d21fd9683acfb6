"""Parts of the workspace that only an output which is not wanted, or the tiles that a call does not take, would read:
nothing is written there."""
import pytest

import vocab_cases as C
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


def _untouched(rows, vocab, width, dtype, **wanted):
    """Bytes that the backward call leaves as they were; its results are those of the whole call."""
    h, table, targets, up = C.problem(rows, vocab, width, dtype, 3)
    lse = L.cross_entropy(h, table, targets, cap=30.0)["lse"]
    whole = L.cross_entropy_backward(h, table, targets, lse, up, cap=30.0)
    need, left = L.cross_entropy_backward_workspace_bytes(rows, vocab, width, dtype), None
    for fill in (0xA5, 0x3C):      # a byte that happens to be written as it was differs the other time
        room = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        got = L.cross_entropy_backward(h, table, targets, lse, up, cap=30.0, workspace=room, **wanted)
        assert all(torch.equal(got[n], whole[n]) for n in got)
        left = room == fill if left is None else left & (room == fill)
    return int(left.sum())


def test_without_the_tables_gradient():
    """Up to 1024 bf16 rows dz's rounding's rest stands behind it, half of dz's part, for the table's gradient alone; and h
    once more."""
    half = 1024 * 20224 * 2 + 1024 * 64 * 2
    assert _untouched(1000, 20000, 64, C.BF16) < half <= _untouched(1000, 20000, 64, C.BF16, want_dtable=False)


def test_sums_of_targets_without_the_tables_gradient():
    """The targets' rests, [rows, width] fp32, and what sorts them."""
    rows, vocab, width = 4100, 2003, 1024
    assert _untouched(rows, vocab, width, C.BF16, want_dtable=False) >= rows * width * 4 + vocab * 4


def test_without_the_rows_gradient():
    """fp32: three planes of the table are for dh alone.  (Up to 32 rows nothing else of it is laid out, past them two planes.)"""
    vocab, width = 20000, 512
    planes = vocab * width * 6
    for rows in (20, 70):
        assert _untouched(rows, vocab, width, C.F32) < planes <= _untouched(rows, vocab, width, C.F32, want_dh=False)


def test_fp32_without_the_tables_gradient():
    """The three planes of h are for the table's gradient alone, past 32 rows."""
    rows, width = 2000, 1024
    assert _untouched(rows, 70, width, C.F32) < rows * width * 6 <= _untouched(rows, 70, width, C.F32, want_dtable=False)
