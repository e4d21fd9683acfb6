"""Shapes of a workgroup that the recurrence's kernels cannot have do not compile (CPU: hipcc's front end only).

In the backward pass one wave passes through the rows, a second rebuilds the states and a third publishes the
tile's span for the tiles after it: with two waves every later tile would wait for ever.  And the walk gives each of a
wave's lanes one channel: a slab of more than 64 would leave some out."""
import os
import subprocess

import pytest

from paper_2506_05233_amd import build as B

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

BACKWARD = "template __global__ void recurrence_grad_kernel<q8_t, bf16_t, true, true, Form<%d>>(RecurrenceGradArgs);"
FORWARD = "template __global__ void recurrence_kernel<bf16_t, true, true, false, Form<%d>>(RecurrenceArgs);"


def _compiles(tmp_path, line):
    src = tmp_path / "form.hip"
    src.write_text('#include "%s"\nnamespace mesa {\nnamespace {\n%s\n}\n}\n' % (os.path.join(B.CSRC, "recurrence.hip"), line))
    res = subprocess.run([HIPCC] + B.HIPCC_FLAGS + ["--cuda-device-only", "-fsyntax-only", str(src)], capture_output=True, text=True)
    return res.returncode == 0, res.stderr


@pytest.mark.parametrize("line,across,reason", [
    (BACKWARD, 16, None), (BACKWARD, 8, None), (BACKWARD, 4, "a wave for each"), (BACKWARD, 32, "a channel in each lane"),
    (FORWARD, 16, None), (FORWARD, 8, None), (FORWARD, 32, "a channel in each lane")])
def test_forms(tmp_path, line, across, reason):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    ok, err = _compiles(tmp_path, line % across)
    assert ok == (reason is None), err[-2000:]
    assert ok or reason in err
