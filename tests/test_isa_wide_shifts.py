"""64-bit shifts by a vector register, checked in the compiled code of every kernel (no
GPU needed).  On this hardware such a shift has given wrong results where the register
that holds the amount is the last one of a wave's allocation and waves share a SIMD.
Registers are allocated in eights."""

import concurrent.futures
import os
import re
import shutil
import subprocess

import pytest

from paper_1904_10584_amd import build

SHIFT = re.compile(r"^\s+v_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)\S*\s+v\[\d+:\d+\],\s*v(\d+),")


def _by_the_last_register(lines):
    """(kernel, instruction) of each shift whose amount is in the last register of the
    kernel's allocation; lines: a compiled source."""
    found, shifts, allocated = [], {}, {}
    name = None
    for line in lines:
        if m := re.match(r"^(\w+):", line):
            name = m.group(1)
        elif line.strip().startswith(".amdhsa_kernel"):
            name = line.split()[1]
        elif m := re.search(r"\.amdhsa_next_free_vgpr (\d+)", line):
            allocated[name] = -(-int(m.group(1)) // 8) * 8
        elif m := SHIFT.match(line):
            shifts.setdefault(name, []).append((int(m.group(1)), line.strip()))
    for k, v in shifts.items():
        found += [(k, text) for amount, text in v if allocated.get(k, 0) == amount + 1 or k not in allocated]
    return found


def _compiled(tmp_path, source):
    out = tmp_path / (source + ".s")
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)]
    p = subprocess.run(cmd, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    # (labels within a kernel start with a dot)
    return out.read_text().split("\n")


def test_no_kernel_shifts_by_its_last_register(tmp_path):
    if not shutil.which(build.HIPCC) and not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    with concurrent.futures.ThreadPoolExecutor(8) as ex:
        texts = list(ex.map(lambda s: _compiled(tmp_path, s), build.SOURCES))
    kernels = 0
    for source, lines in zip(build.SOURCES, texts):
        kernels += sum(".amdhsa_next_free_vgpr" in line for line in lines)
        assert not _by_the_last_register(lines), source
    assert kernels > 100


def test_the_search_finds_one():
    text = ["k:", "\tv_lshrrev_b64 v[8:9], v39, v[4:5]", "\t.amdhsa_kernel k", "\t\t.amdhsa_next_free_vgpr 40"]
    assert len(_by_the_last_register(text)) == 1
    assert not _by_the_last_register(text[:-1] + ["\t\t.amdhsa_next_free_vgpr 41"])
    assert not _by_the_last_register(["k:", "\tv_lshrrev_b64 v[8:9], 16, v[4:5]"] + text[2:])
