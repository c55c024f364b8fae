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


# ---- numbers past the range of their type ----------------------------------------------------------------------------------------

def test_numbers_past_the_range_of_their_type(p):
    """No sequences, so that nothing is launched: what is taken returns 0.  A number that its C type does not hold is refused, and not taken by its low bits."""
    n, P = p._ns(), Ptr()
    append = lambda old, new, B=0, n_in=3, sb=8: n.vfa_kv8_append_t(P, P, P, P, P, P, B, 2, 128, n_in, 64, sb, 8, 8, 8, 8, 8, None, None, old, new, 0)
    read = lambda length, B=0: n.vfa_kv8_read_t(P, P, P, P, P, P, B, 2, 128, 3, 64, None, length, 0)
    decode = lambda n_keys, B=0, ns=1, size=0: n.vfa_kv8_decode_fwd_t(P, P, P, P, P, P, P, B, 4, 2, 128, 1, 64, None, n_keys, ns, 0.0, None, size, 0)
    rope = lambda first, B=0, sb=8: n.vfa_qk_norm_rope_fwd_t(P, P, P, P, P, P, B, 3, 4, 2, 64, sb, 8, 8, 8, 8, 8, 8, 8, 8, 1, None, None, 1e-6, P, 4, 64, 0, None, first, 0)
    assert append(0, 3) == 0 and read(5) == 0 and decode(5) == 0 and rope(2) == 0 and rope(-2 ** 31) == 0 and read(2 ** 31 - 1) == 0
    for big in (2 ** 31, 2 ** 32, 2 ** 32 + 3, 2 ** 63, 2 ** 64 + 3, 10 ** 30, -2 ** 31 - 1, -2 ** 32, -10 ** 30):
        assert append(0, big) == -1 and append(big, 3) == -1 and read(big) == -1 and decode(big) == -1 and rope(big) == -1
        assert append(0, 3, B=big) == -1 and read(5, B=big) == -1 and decode(5, B=big) == -1 and rope(2, B=big) == -1
        assert append(0, 3, n_in=big) == -1 and decode(5, ns=big) == -1
    for big in (2 ** 63, 2 ** 64 + 8, -2 ** 63 - 8):
        assert append(0, 3, sb=big) == -1 and rope(2, sb=big) == -1
    assert append(0, 3, sb=2 ** 62) == 0 and decode(5, size=2 ** 64 - 1) == 0 and decode(5, size=2 ** 64) == -1 and decode(5, size=-1) == -1
    for bad in (None, "3", [3]):
        with pytest.raises(TypeError):
            decode(bad)
    assert n.vfa_kv8_decode_splits(2 ** 32 + 1, 4, 2, 1, 64, 4096, 0) == 1 and n.vfa_kv8_decode_splits(1, 4, 2, 1, 64, 2 ** 32 + 4096, 0) == 1
    assert n.vfa_kv8_decode_workspace_bytes(2 ** 32 + 1, 4, 1, 64, 3) == 0


class Ptr:
    def data_ptr(self):
        return 0x1000


def test_suggested_ranges_at_the_end_of_the_type(p):
    """Lengths above the largest that fits whole blocks into an int are as that."""
    L = p.lib()
    most = 2 ** 31 - 64
    for B, Hq, Hkv, n_q in ((1, 8, 8, 1), (1, 32, 8, 1), (4, 32, 8, 1), (1, 32, 8, 4), (1, 32, 8, 64), (16, 32, 8, 1), (1, 1, 1, 1)):
        for d in (64, 128):
            for varlen in (0, 1):
                want = L.vfa_kv8_decode_splits(B, Hq, Hkv, n_q, d, most, varlen)
                for n in (most + 1, most + 2, 2 ** 31 - 1):
                    assert L.vfa_kv8_decode_splits(B, Hq, Hkv, n_q, d, n, varlen) == want, (B, Hq, Hkv, n_q, d, varlen, n)
