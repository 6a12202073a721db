"""The stream that a call without one goes to: torch's current stream, by whichever
of torch's ways to it there is (no GPU needed)."""

import types

import pytest
import torch

from paper_1904_10584_amd import binding as am


def _handle(s):
    return getattr(s, "value", s)  # (ctypes takes either)


@pytest.fixture
def two_ways(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x1230))
    monkeypatch.setattr(am, "_raw_device", lambda: 5)
    monkeypatch.setattr(am, "_raw_stream", lambda device: 0x4560 + device)


def test_a_given_stream(two_ways):
    assert _handle(am._stream(types.SimpleNamespace(cuda_stream=0x7890))) == 0x7890


def test_the_raw_handle(two_ways):
    assert _handle(am._stream(None)) == 0x4565


@pytest.mark.parametrize("missing", ["_raw_stream", "_raw_device"])
def test_a_torch_without_raw_handles(two_ways, monkeypatch, missing):
    monkeypatch.setattr(am, missing, None)
    assert _handle(am._stream(None)) == 0x1230


def test_before_torch_has_a_device(two_ways, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    assert _handle(am._stream(None)) == 0x1230


def test_names_that_are_missing_are_found_out_when_the_module_loads(monkeypatch):
    import importlib.util
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    spec = importlib.util.spec_from_file_location("paper_1904_10584_amd._binding_again", am.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    assert again._raw_stream is None
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x1230))
    assert _handle(again._stream(None)) == 0x1230
