"""The binding of the operators beside the cache, on the host: first calls from several threads, and what it refuses by itself."""
import sys

import pytest

from paper_2609_14507_b200 import binding

torch = pytest.importorskip("torch")


def fresh(monkeypatch):
    """As before the first call."""
    names = [n for n in ("_torch", "_np", "_bf16", "_f32", "_i32", "_int64", "_int32", "_current_device", "_current_stream") if hasattr(binding, n)]
    for n in names:
        monkeypatch.setattr(binding, n, None)
    return names


def test_a_call_that_finds_the_modules_finds_all_of_them(monkeypatch):
    """The entry points look at one name to know whether the others are there: whichever line of the first call another thread
    interrupts, that name comes last."""
    names = fresh(monkeypatch)
    seen = []

    def trace(frame, event, arg):
        if frame.f_code is binding._modules.__code__:
            seen.append((binding._torch is not None, [n for n in names if getattr(binding, n) is None]))
        return trace

    sys.settrace(trace)
    try:
        binding._modules()
    finally:
        sys.settrace(None)
    assert seen and binding._torch is torch
    assert all(not missing for there, missing in seen if there)
