"""Sizes at which 64 bits or a launch would end: the gated delta rule's workspace query and
8-bit matrices, on the host."""

import ctypes

import pytest

from paper_1904_10584_amd import binding as am

P = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first


@pytest.mark.parametrize("T,B,heads,varlen,train", [
    (1 << 30, 1, 1 << 22, 0, 1), (1 << 30, 3, 1 << 20, 0, 1), (1 << 20, 1 << 11, 1 << 19, 0, 1),
    (64, 1 << 12, 1 << 12, 0, 1), (1, 1 << 12, 1 << 11, 0, 0), (1, 1, (1 << 31) - 1, 0, 0),
    ((1 << 31) - 1, 1, 1, 0, 0), (1 << 20, 1 << 11, 1, 0, 0), (5, 1025, 1, 1, 0),
    ((1 << 20) - 1, 1 << 9, 1, 0, 1)])
def test_sizes_that_a_call_refuses_have_no_workspace(T, B, heads, varlen, train):
    """(Some of these passed 2^63 bytes and came back as other numbers.)"""
    L = am.lib()
    assert L.am_gated_delta_workspace_bytes(T, B, heads, heads, 128, 128, am.BF16, varlen, train) == -1
    lens = (ctypes.c_int32 * B)(*[T] * B) if varlen else None
    wide = 1 << 40
    st = L.gated_delta_forward(T, B, heads, heads, 128, 128, am.BF16, lens, P, wide, P, wide, P, wide, P, wide, P, wide,
                               P, 8.0, 1e-6, None, P, wide, None, train, P, 1 << 62, None)
    assert st == am.EUNSUPPORTED, L.am_last_error()


@pytest.mark.parametrize("T,B,heads,varlen,train", [
    (1, (1 << 23) - 1, 1, 0, 0), (1 << 30, 1, 1, 0, 0), ((1 << 20) - 1, (1 << 9) - 1, 1, 0, 1), (1 << 20, 1024, 2, 1, 0)])
def test_the_largest_sizes_have_one(T, B, heads, varlen, train):
    chunks = -(-T // 64)
    kept = (2 * chunks - 1) * B * heads * 128 * 128 * 4 if train else 0
    n = am.lib().am_gated_delta_workspace_bytes(T, B, heads, heads, 128, 128, am.BF16, varlen, train)
    assert kept <= n < 1 << 50
