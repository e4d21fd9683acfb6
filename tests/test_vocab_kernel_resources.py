"""Registers of the embedding's and the cross entropy's kernels, from the compiler's resource report (CPU;
tests/test_kernel_resources.py reads the same report for spills in every source)."""
import concurrent.futures
import os
import re

import pytest

import test_kernel_resources as K
from paper_2506_05233_amd import build as B

SOURCES = ("embedding.hip", "cross_entropy.hip")


@pytest.fixture(scope="module")
def reports():
    if not os.path.exists(K.HIPCC) or K._demangler() is None:
        pytest.skip("hipcc or a C++ demangler is not available")
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        merged = {k: v for r in ex.map(K._report, [os.path.join(B.CSRC, s) for s in SOURCES]) for k, v in r.items()}
    names = K._demangle(sorted(merged))
    return {names[k].replace("mesa::", "").replace("(anonymous namespace)::", ""): v for k, v in merged.items()}


# name, registers a lane at most: 256 for one workgroup of 512 threads on a compute unit (two waves a SIMD), 168 for
# three waves a SIMD, 128 for four, 96 for five.  The tiles' costs were measured with them.
LIMITS = [
    (r"logits(_grad)?_kernel<TileShape<1, 256, 256, 2, 4>", 256),
    (r"(logits|logits_grad|grad)_kernel<TileShape<1, 128, 128, 2, 2>", 256),
    (r"(logits|logits_grad|grad)_kernel<TileShape<(1|2|3), 64, 64, ", 128),
    (r"(logits|logits_grad|grad)_kernel<TileShape<1, 64, 32, ", 128),
    (r"(logits|logits_grad)_kernel<TileShape<2, 64, 32, ", 168),
    (r"grad_kernel<TileShape<1, 256, 256, 2, 4>", 256),
    (r"(logits|logits_grad)_kernel<TileShape<2, ", 256),
    (r"grad_kernel<TileShape<3, ", 256),
    (r"join_kernel<(1|16)>", 64),
    (r"pack_(copy|rows)_kernel", 96),
    (r"embedding_kernel<(float|bf16_t), (float|bf16_t), (1|8), (1|2)>", 64),
    (r"token_(histogram|scatter)_kernel", 64),
    (r"token_sort_kernel<(1|2)>", 64),
    (r"token_piece_kernel<float, (float|bf16_t), 8, (8|16)>", 256),
    (r"token_piece_kernel<bf16_t, (float|bf16_t), 8, (8|16)>", 168),
    (r"token_run_kernel", 168),
    (r"token_join_kernel", 256),
]


@pytest.mark.parametrize("pattern,most", LIMITS)
def test_registers(reports, pattern, most):
    found = [(n, r) for n, r in reports.items() if re.search(pattern, n)]
    assert found, pattern
    for n, r in found:
        assert r["VGPRs"] + r.get("AGPRs", 0) <= most, (n, r["VGPRs"])
        assert r.get("VGPRs Spill", 0) == 0 and r.get("ScratchSize [bytes/lane]", 0) == 0, n
