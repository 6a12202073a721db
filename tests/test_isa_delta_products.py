"""The gated delta rule's matrix instructions, checked in the compiled code (no GPU
needed).  One of 16 elements of the sum that adds to what one of 32 has just written gave
wrong sums on this hardware: the kernels have the form of 32 alone."""

import concurrent.futures
import os
import re
import shutil
import subprocess

import pytest

from paper_1904_10584_amd import build


def _products(tmp_path, source):
    out = tmp_path / (source + ".s")
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)]
    p = subprocess.run(cmd, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    return set(re.findall(r"\bv_mfma_\w+", out.read_text()))


def test_products_have_one_form(tmp_path):
    if not shutil.which(build.HIPCC) and not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        found = list(ex.map(lambda s: _products(tmp_path, s), ["gated_delta.hip", "gated_delta_backward.hip"]))
    assert found == [{"v_mfma_f32_16x16x32_bf16"}] * 2
