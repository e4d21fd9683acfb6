"""Sizes at the end of what one launch holds, on the GPU."""
import pytest

from paper_2506_05233_amd import libmesa as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    L.load()
    yield
    torch.cuda.empty_cache()


def test_one_token_of_many_sequences():
    """The last batch that fits one launch of 512 threads a sequence is right to its end, the next is refused."""
    for B, fits in (((1 << 23) - 1, True), (1 << 23, False)):
        x = torch.ones((B, 1, 4), device="cuda")
        th = torch.full((4,), -3.0, device="cuda")
        out = torch.full_like(x, 7.0)
        if fits:
            L.recurrence(x, x, x, th, out=out)
            assert bool((out == out[0]).all()) and 0.0 < float(out[0, 0, 0]) < 1.0
        else:
            with pytest.raises(L.MesaError) as e:
                L.recurrence(x, x, x, th, out=out)
            assert e.value.status == L.MESA_ERR_SHAPE and bool((out == 7.0).all())


def test_state_of_an_empty_sequence_past_32_bits():
    """2^32 states and more are handed on whole when there is no token (17 GB, written as zeros)."""
    B, W = (1 << 22) + 1, 1024
    final = torch.ones(B * W, device="cuda")
    st = L.load().mesa_recurrence(None, None, None, None, 8.0, None, None, B, 0, W, W, 0, None, final.data_ptr(), None, None, None,
                                  None, None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == L.MESA_OK
    assert not bool(final.view(-1, W).any(dim=1).any())


def test_packed_states_past_32_bits():
    """More state elements than a launch has threads: the last pairs are converted as the first."""
    pairs, d = (1 << 18) + 3, 128
    full = torch.zeros((pairs, 1, d, d), device="cuda")
    for p in (0, 1, pairs - 2, pairs - 1):
        a = torch.randn((d, d), generator=torch.Generator().manual_seed(p)).cuda()
        full[p, 0] = a + a.T
    packed = L.pack_state(full)
    few = torch.cat([full[:2], full[-2:]])
    want = L.pack_state(few)
    assert torch.equal(torch.cat([packed[:2], packed[-2:]]), want) and not bool(packed[2:-2].any())
    del full
    back = L.unpack_state(packed)
    assert torch.equal(torch.cat([back[:2], back[-2:]]), few) and not bool(back[2:-2].any())
