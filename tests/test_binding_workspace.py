"""The workspace that a caller hands to the binding: kernels write all the bytes that it counts, so it has to hold
them.  (The helper is asked on CPU tensors; nothing is launched.)"""
import pytest

from paper_2506_05233_amd import libmesa as L

torch = pytest.importorskip("torch")

CPU = torch.device("cpu")


def test_a_workspace_that_holds_its_bytes_is_used():
    for ws in (torch.empty(4096, dtype=torch.uint8), torch.empty(1024), torch.empty((4, 8, 16, 8), dtype=torch.uint8)):
        assert L._workspace(ws, 4096, CPU) is ws


def test_one_that_is_too_small_or_elsewhere_is_replaced():
    for ws in (None, torch.empty(4095, dtype=torch.uint8), torch.empty(0), torch.empty(4096, dtype=torch.uint8, device="meta")):
        got = L._workspace(ws, 4096, CPU)
        assert got is not ws and got.device == CPU and got.numel() * got.element_size() >= 4096 and got.is_contiguous()
    assert L._workspace(None, 0, CPU) is None


@pytest.mark.parametrize("ws", [torch.empty(1, dtype=torch.uint8).expand(4096), torch.empty(8192, dtype=torch.uint8)[::2],
                                torch.empty((64, 128), dtype=torch.uint8).t(), torch.empty((64, 128), dtype=torch.uint8)[:, :64]])
def test_a_view_that_does_not_hold_them_is_refused(ws):
    """One byte counted 4096 times, every other byte of a tensor, another order, a slice of rows."""
    with pytest.raises(ValueError):
        L._workspace(ws, 4096, CPU)


def test_not_a_tensor():
    with pytest.raises(TypeError):
        L._workspace(bytearray(4096), 4096, CPU)
