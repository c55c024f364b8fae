"""What the Python wrappers of the serving operators do around a call: first calls from two threads, numbers past the range of their type, suggestions.  CPU
only: calls that have nothing to do."""
import os
import sys

import pytest

from paper_2604_12798_amd import build


@pytest.fixture(scope="module")
def p():
    import paper_2604_12798_amd as pkg
    if not os.path.exists(pkg.LIB_PATH) or not os.path.exists(build.BINDING):
        build.build_lib()
    pkg._ns()
    return pkg


def test_all_names_are_there_before_another_thread_may_use_one(p, monkeypatch):
    """Line by line through the first call: a thread that comes in between either makes the names itself or finds all of them."""
    names = ("_empty_like", "_f32", "_u8", "_current_device", "_current_stream")
    for n in names:
        monkeypatch.setattr(p, n, None)
    seen = []

    def trace(frame, event, arg):
        if frame.f_code is p._ns.__code__:
            missing = [n for n in names if getattr(p, n) is None]
            seen.append((p._empty_like is not None, missing))
            return trace
        return None

    old = sys.gettrace()
    sys.settrace(trace)
    try:
        p._ns()
    finally:
        sys.settrace(old)
    assert seen[0] == (False, list(names)) and seen[-1] == (True, [])
    assert all(not there or not missing for there, missing in seen), seen
