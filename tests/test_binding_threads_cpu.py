"""What the binding looks up once: a thread that comes while another is at it finds all of it or nothing (no GPU needed)."""
import sys

import pytest
import torch

from paper_2006_02924_amd import binding as B


@pytest.mark.parametrize("torch_has_it", [True, False])
def test_streams_are_looked_up_whole(monkeypatch, torch_has_it):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    if torch_has_it:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(B, "_current_device", None)
    monkeypatch.setattr(B, "_current_stream", None)
    seen = []

    def trace(frame, event, arg):
        if frame.f_code is B._learn_streams.__code__:
            # (what another thread would find between two lines)
            seen.append(B._current_device is None or B._current_device() == -1 or B._current_stream is not None)
            return trace
        return None

    old = sys.gettrace()
    sys.settrace(trace)
    try:
        B._learn_streams()
    finally:
        sys.settrace(old)
    assert len(seen) > 3 and all(seen)
    assert B._current_device() == (0 if torch_has_it else -1) and (B._current_stream is not None) == torch_has_it
