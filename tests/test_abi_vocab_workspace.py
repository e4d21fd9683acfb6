"""What the cross entropy's backward pass may ask for, as include/libmesa.h states it (CPU: the queries launch nothing)."""
import os

import pytest

from paper_2506_05233_amd import libmesa as L

F32, BF16 = L.MESA_DTYPE_F32, L.MESA_DTYPE_BF16
MIB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(L.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    L.load()


def _stated(rows, vocab, width, dtype):
    """The header's bound, in bytes: copies of the rows and fp32 sums of them (rows and width filled up to 64), the copy of a part of the
    table, dz of that part, and two times sums of layers; and what the sorted targets and the table's exponents take."""
    r, w = -(-rows // 64) * 64, -(-width // 64) * 64
    least = 256 * w * (2 if dtype == BF16 else 10)
    dz = max(1 << 27, 512 * r) * (2 if dtype == BF16 else 6)
    return 10 * r * w + max(1024 * MIB, least) + dz + 256 * MIB + max(256 * MIB, r * w * 4) + 32 * r + 8 * vocab + MIB


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bound(dtype):
    for rows in (1, 3, 32, 33, 256, 1000, 1025, 4000, 16384, 100000):
        for vocab in (1, 5003, 50257, 131072, 1 << 20):
            for width in (1, 64, 1000, 2048, 4096, 65536):
                need = L.cross_entropy_backward_workspace_bytes(rows, vocab, width, dtype)
                assert 0 < need <= _stated(rows, vocab, width, dtype), (rows, vocab, width, need / MIB, _stated(rows, vocab, width, dtype) / MIB)


@pytest.mark.parametrize("rows,vocab,width,dtype,most", [
    (1, 50257, 2048, F32, 620), (32, 50257, 2048, F32, 640), (256, 131072, 4096, F32, 1330), (1, 128000, 4096, BF16, 1040), (256, 50257, 2048, BF16, 350)])
def test_few_rows(rows, vocab, width, dtype, most):
    """Of fp32 no more of the table than its three planes, and no more than 1 GiB of it."""
    assert L.cross_entropy_backward_workspace_bytes(rows, vocab, width, dtype) <= most * MIB


def test_few_fp32_rows_forward():
    """Three planes of h, the tiles' sums, and nothing of the two planes that more rows take."""
    for rows, vocab in ((1, 50), (32, 50), (32, 50257)):
        tiles = -(-vocab // 64)
        assert L.cross_entropy_workspace_bytes(rows, vocab, 65536, F32) <= rows * 65536 * 6 + 16 * rows * tiles + 4 * rows + 2048
