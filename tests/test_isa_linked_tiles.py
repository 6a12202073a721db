"""The words that link the gated recurrence's tiles, checked in the compiled code
(no GPU needed).  XCDs do not share their L2s: what one tile publishes and another
reads must carry the agent scope (sc1), and a tile's flag may leave only after its
stores have arrived."""

import os
import re
import shutil
import subprocess

import pytest

from paper_1904_10584_amd import build


def _kernels(tmp_path):
    if not shutil.which(build.HIPCC) and not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = tmp_path / "gated_recurrence.s"
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S",
           os.path.join(build.CSRC, "gated_recurrence.hip"), "-o", str(out)]
    p = subprocess.run(cmd, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    name, body = None, []
    for line in out.read_text().split("\n"):
        head = re.match(r"^(_Z\S*gr_(?:forward|backward)_kernel\S*):", line)
        if head:
            name, body = head.group(1), []
        elif name and line.startswith(".Lfunc_end"):
            yield name, body
            name = None
        elif name:
            body.append(line.split(";")[0].strip())


def test_links_carry_the_agent_scope_and_flags_wait(tmp_path):
    linked = 0
    for name, body in _kernels(tmp_path):
        scoped = [s for s in body if re.search(r"\bsc1\b", s)]
        if "TilesE2" not in name:  # (Tiles::LINKED)
            assert not scoped, name
            continue
        linked += 1
        pairs = 2 if "Li2E" in name else 1  # channels of a lane: words of 64 bits
        loads = [s for s in scoped if s.startswith("global_load")]
        # flags by the word; parts of two tiles and the block's start
        assert any(s.startswith("global_load_dword ") for s in loads), name
        words = sum(2 if "dwordx4" in s else 1 for s in loads if "dwordx2" in s or "dwordx4" in s)
        assert words >= 3 * pairs, (name, loads)
        # a tile's pairs and then its flag, after a wait for all of them; a block's states
        events = []
        for s in body:
            if re.match(r"global_store_dwordx[24] .*\bsc1\b", s):
                events.append("pair")
            elif re.match(r"global_store_dword .*\bsc1\b", s):
                events.append("flag")
            elif s.startswith("s_waitcnt") and re.search(r"vmcnt\(0\)", s):
                events.append("wait")
        flags = [k for k, e in enumerate(events) if e == "flag"]
        assert len(flags) == 1 and "pair" in events[:flags[0]] and "pair" in events[flags[0]:], (name, events)
        assert events[flags[0] - 1] == "wait", (name, events)
    assert linked == 12
