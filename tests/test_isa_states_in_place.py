"""States that are updated in place (hT over h0, dh0 over dhT), checked in the
compiled code (no GPU needed).  One wave of a workgroup stores the new state, every
wave loads the old one: a wave's load has to be back before the barrier that the
storing wave passes.  That barrier waits for LDS alone, so a wait for the load
stands before it in every kernel of several waves."""

import os
import re
import shutil
import subprocess

import pytest

from paper_1904_10584_amd import build


def _unfinished(body, before_frames=False):
    """Of the ordinary loads of the text, those of the states and of the channels'
    rates among them, the ones that may still be in flight at the first barrier
    after the first of the frames' loads (through buffer descriptors).  Loads come
    back in their order; vmcnt(n) waits for all but the last n operations.
    before_frames: only of those before the frames' loads, two at least (the
    backward pass loads its start and the rates there, and after them the states
    that the forward pass saved, which nothing updates in place)."""
    flying, frames, early = [], False, 0
    for line in body:
        s = line.split(";")[0].strip()
        if re.match(r"(global|buffer|flat|scratch)_(load|store|atomic)", s):
            frames = frames or s.startswith("buffer_load")
            ordinary = re.match(r"(global|flat)_load", s) is not None
            early += ordinary and not frames
            flying.append((ordinary and not (before_frames and frames), s))
        elif s.startswith("s_waitcnt") and "vmcnt" in s:
            n = int(re.search(r"vmcnt\((\d+)\)", s).group(1))
            flying = flying[len(flying) - min(n, len(flying)):]
        elif s.startswith("s_barrier") and frames:
            assert early >= 2 or not before_frames
            return [f for counts, f in flying if counts]
    return None


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
            body.append(line)


def test_every_wave_has_read_its_start_at_the_first_barrier(tmp_path):
    seen = 0
    for name, body in _kernels(tmp_path):
        late = _unfinished(body, before_frames="gr_backward" in name)
        if late is None:  # (one wave: no barrier)
            assert "ELi1ELi1EEE" in name, name
            continue
        seen += 1
        assert not late, (name, late)
    assert seen == 6 * 3 + 6 * 2  # forward: in turn, linked, one tile; backward: in turn, linked


def test_the_walk_finds_a_load_in_flight():
    frames, old = "buffer_load_dword v1, v0, s[0:3], 0 offen", "global_load_dword v9, v[2:3], off"
    barrier = "s_barrier"
    assert _unfinished([frames, old, "s_waitcnt lgkmcnt(0)", barrier]) == [old]
    assert _unfinished([old, frames, "s_waitcnt vmcnt(1)", barrier]) == []
    assert _unfinished([frames, old, "s_waitcnt vmcnt(1)", barrier]) == [old]
    assert _unfinished([frames, old, "s_waitcnt vmcnt(0)", barrier]) == []
    assert _unfinished([old]) is None
    assert _unfinished([old, old, frames, old, "s_waitcnt vmcnt(2)", barrier], before_frames=True) == []
    assert _unfinished([old, old, frames, "s_waitcnt vmcnt(2)", barrier], before_frames=True) == [old]
