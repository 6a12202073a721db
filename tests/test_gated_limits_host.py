"""Sizes at the ends of what the gated recurrence's kernels can count, on the host."""

import ctypes

import pytest

from paper_1904_10584_amd import binding as am

P = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first


def _forward(T, lengths=None):
    lp = None if lengths is None else (ctypes.c_int32 * len(lengths))(*lengths)
    L = am.lib()
    # (no workspace: a size that is accepted is refused for that, and nothing is enqueued)
    st = L.gated_recurrence_forward(T, 1 if lp is None else len(lengths), 2, am.F32, lp, P, P, P, 2, P, 8.0, None, P,
                                    None, 0, None, 0, None)
    return st, L.am_last_error().decode()


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 128, 2 ** 31 - 256])
def test_frames_that_would_pass_32_bits_at_a_tiles_end_are_refused(T):
    """The last tile's frames are counted to its end, 127 past the last frame, and
    the schedule's to the end of its last workgroup: both in 32 bits."""
    for lengths in (None, [T]):
        st, msg = _forward(T, lengths)
        assert st == am.EUNSUPPORTED and "frames" in msg


def test_the_longest_sequence_is_taken():
    T = 2 ** 31 - 257
    assert T + 256 < 2 ** 31
    for lengths in (None, [T], [T, 0]):
        st, msg = _forward(T, lengths)
        assert st == am.EWORKSPACE, msg
