"""Registers of the recurrence's, the checkpoints' and the ends' gradients' kernels, from the compiler's resource
report (CPU; tests/test_kernel_resources.py reads the same report for spills in every source)."""
import concurrent.futures
import os
import re

import pytest

import test_kernel_resources as K
from paper_2506_05233_amd import build as B

SOURCES = ("recurrence.hip", "checkpoint.hip", "layer_ends_grad.hip")


@pytest.fixture(scope="module")
def reports():
    if not os.path.exists(K.HIPCC) or K._demangler() is None:
        pytest.skip("hipcc or a C++ demangler is not available")
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        merged = {k: v for r in ex.map(K._report, [os.path.join(B.CSRC, s) for s in SOURCES]) for k, v in r.items()}
    names = K._demangle(sorted(merged))
    return {names[k].replace("mesa::", "").replace("(anonymous namespace)::", ""): v for k, v in merged.items()}


def test_every_kernel_is_reported(reports):
    for k in ("recurrence_kernel", "recurrence_grad_kernel", "recurrence_step_kernel", "recurrence_fill_kernel", "recurrence_dtheta_kernel",
              "recurrence_copy_kernel", "checkpoint_pack_kernel", "checkpoint_unpack_kernel", "frontend_grad_kernel",
              "output_norm_grad_kernel", "partial_sum_kernel"):
        assert any(k in name for name in reports), k


# name, registers a lane at most: 128 leave room for two workgroups of 512 threads on a compute unit (four waves a
# SIMD), 256 for one; 168 for three waves a SIMD, 72 for seven.  Where a kernel is built for the former the figures
# beside it were measured with it.
LIMITS = [
    (r"recurrence_kernel<(float|bf16_t), true, (true|false), (true|false), Form<(8|16)>", 128),
    (r"recurrence_grad_kernel<(bf16_t|q8_t), bf16_t, (true|false), (true|false), Form<(8|16)>", 128),
    (r"recurrence_grad_kernel<(float|bf16_t|q8_t), float, (true|false), (true|false), Form<(8|16)>", 256),
    (r"recurrence_step_kernel<(float|bf16_t), (1|4)>", 64),
    (r"checkpoint_(pack|unpack)_kernel<(float|bf16_t), (true|false)>", 64),
    (r"frontend_grad_kernel<(float|bf16_t|q8_t), (float|bf16_t), (64|128), (64|128)>", 168),
    (r"output_norm_grad_kernel<(float|q8_t), (float|bf16_t), (64|128)>", 72),
]


@pytest.mark.parametrize("pattern,most", LIMITS)
def test_registers_leave_the_workgroups_that_a_kernel_is_built_for(reports, pattern, most):
    found = [(n, r) for n, r in reports.items() if re.search(pattern, n)]
    assert found, pattern
    for n, r in found:
        assert r["VGPRs"] + r.get("AGPRs", 0) <= most, (n, r["VGPRs"])
        assert r.get("VGPRs Spill", 0) == 0 and r.get("ScratchSize [bytes/lane]", 0) == 0, n
