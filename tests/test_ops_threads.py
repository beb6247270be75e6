"""CPU test of the operators' binding: threads whose first calls meet."""
import importlib.util
import sys
import threading

import pytest
import torch

A = pytest.importorskip("paper_2504_13850_amd.api")


def _met_at_line(count):
    """The first call of a freshly loaded binding, with another thread's first call at its line number `count` (counted
    in the order of execution).  Returns the other thread's errors and the lines that were run."""
    spec = importlib.util.spec_from_file_location("paper_2504_13850_amd.api_first_call", A.__file__)
    fresh = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(fresh)
    t, i = torch.zeros((4, 2, 8), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    errors, lines = [], []

    def make():
        try:
            fresh.make_attn(t, t, t, t, i, i, i, i, 4, 4)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    def at_line(frame, event, arg):
        if event == "line":
            if len(lines) == count:
                other = threading.Thread(target=make)
                other.start()
                other.join()
            lines.append(frame.f_lineno)
        return at_line

    def at_call(frame, event, arg):
        return at_line if frame.f_code.co_filename == A.__file__ else None

    before = sys.gettrace()
    sys.settrace(at_call)
    try:
        fresh.make_attn(t, t, t, t, i, i, i, i, 4, 4)
    finally:
        sys.settrace(before)
    return errors, lines


def test_first_calls_of_two_threads():
    _, lines = _met_at_line(-1)
    assert len(lines) > 10
    for n in range(len(lines)):
        errors, _ = _met_at_line(n)
        assert not errors, f"at line {lines[n]}: {errors}"
