"""What the paged cache's operators and masked attention refuse, before anything is launched.  CPU only."""
import ctypes
import os

import pytest

from paper_2604_12798_amd import build
from test_serving_binding import BF, F32, I32, Fake

OK, INVALID, UNSUPPORTED = 0, -1, -2
P, ODD, NONE = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002), ctypes.c_void_p(0)  # never dereferenced
FOUR = ctypes.c_void_p(0x1004)


@pytest.fixture(scope="module")
def p():
    import paper_2604_12798_amd as pkg
    if not os.path.exists(pkg.LIB_PATH) or not os.path.exists(build.BINDING):
        build.build_lib()
    pkg._ns()
    return pkg


def call(f, good, **changed):
    assert set(changed) <= set(good), changed
    return f(*{**good, **changed}.values())


def test_append(p):
    good = dict(K=P, V=P, KP=P, VP=P, table=P, B=1, Hkv=2, n_pages=9, page=16, M=8, n_in=4, d=64, kb=1, kh=8, kn=8, vb=8, vh=8, vn=8, ol=NONE, nl=NONE,
                old=0, new=4, stream=NONE)
    f = p.lib().vfa_kvp_append
    assert call(f, good) == INVALID  # (a stride of 1: no variation below can get as far as a launch)
    assert call(f, good, B=0) == OK and call(f, good, n_in=0, new=0) == OK and call(f, good, old=4) == OK
    assert call(f, good, M=0, new=0) == OK and call(f, good, n_pages=0, KP=NONE, VP=NONE) == OK
    for bad in (dict(B=-1), dict(Hkv=0), dict(n_pages=-1), dict(page=0), dict(page=-16), dict(M=-1), dict(n_in=-1), dict(d=-1), dict(old=-1), dict(old=5), dict(new=129),
                dict(new=5), dict(ol=P), dict(nl=P), dict(ol=ODD, nl=P), dict(ol=P, nl=ODD)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    for bad in (dict(d=96), dict(page=8), dict(page=48), dict(page=17), dict(M=(1 << 26) + 1), dict(page=1 << 30, M=2)):
        assert call(f, good, **{"B": 0, **bad}) == UNSUPPORTED, bad
    for bad in (dict(Hkv=40000), dict(B=40000, Hkv=2)):
        assert call(f, good, **bad) == UNSUPPORTED, bad
    ok = dict(kb=8)
    for bad in (dict(K=NONE), dict(V=NONE), dict(KP=NONE), dict(VP=NONE), dict(table=NONE), dict(K=ODD), dict(V=ODD), dict(KP=FOUR), dict(VP=ODD), dict(table=ODD)):
        assert call(f, good, **ok, **bad) == INVALID, bad
    for name in ("kh", "kn", "vb", "vh", "vn"):
        assert call(f, good, **ok, **{name: 4}) == INVALID


def test_decode(p):
    good = dict(Q=P, KP=P, VP=P, table=P, O=NONE, LSE=NONE, B=1, Hq=4, Hkv=2, n_pages=9, page=16, M=8, n_q=1, d=64, lens=NONE, n_keys=4, ns=1, scale=0.0, cap=0.0,
                slopes=NONE, ws=NONE, wsb=0, stream=NONE)
    f = p.lib().vfa_kvp_decode_fwd
    assert call(f, good) == INVALID  # (no output: no variation below can get as far as a launch)
    assert call(f, good, B=0) == OK and call(f, good, n_q=0) == OK
    nan, inf = float("nan"), float("inf")
    for bad in (dict(B=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(n_q=-1), dict(ns=0), dict(ns=4097), dict(scale=nan), dict(scale=inf), dict(cap=-1.0), dict(cap=nan),
                dict(cap=inf), dict(cap=1e-4), dict(cap=1001.0), dict(slopes=ODD), dict(lens=ODD), dict(n_keys=-1), dict(n_keys=129), dict(page=0), dict(M=-1), dict(n_pages=-1)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    for bad in (dict(d=96), dict(page=8), dict(page=24), dict(Hq=66), dict(M=1 << 27)):
        assert call(f, good, **{"B": 0, **bad}) == UNSUPPORTED, bad
    assert call(f, good, B=0, cap=0.001) == OK and call(f, good, B=0, cap=1000.0) == OK
    for bad in (dict(Q=NONE), dict(Q=ODD), dict(O=ODD), dict(KP=NONE), dict(VP=FOUR), dict(table=NONE), dict(table=ODD), dict(LSE=ODD)):
        assert call(f, good, **{"O": P, **bad}) == INVALID, bad
    many = dict(O=P, ns=2)
    need = p.kvp_decode_workspace_bytes(1, 4, 1, 64, 2)
    for bad in (dict(ws=NONE, wsb=need), dict(ws=ODD, wsb=need), dict(ws=P, wsb=need - 1)):
        assert call(f, good, **many, **bad) == INVALID, bad
    for bad in (dict(B=40000), dict(Hq=2, B=1 << 14, n_q=1 << 17), dict(n_q=1 << 22)):
        assert call(f, good, O=P, **bad) == UNSUPPORTED, bad


def test_decode_helpers(p):
    assert p.kvp_decode_workspace_bytes(2, 4, 1, 64, 3) == (2 * 4 * 3 * 66 * 4 + 16 + 255) // 256 * 256
    assert p.kvp_decode_workspace_bytes(0, 4, 1, 64, 3) == 0 and p.kvp_decode_workspace_bytes(2, 4, 1, 64, 0) == 0
    for args in ((0, 4, 2, 1, 64, 100), (1, 4, 2, 1, 64, 0), (1, 4, 2, 1, 64, 50), (40000, 4, 2, 1, 64, 100000)):
        assert p.kvp_decode_splits(*args) == 1
    for d in (64, 128):
        for varlen in (False, True):
            for n in (1, 1000, 32768, 2 ** 31 - 1):
                for n_q in (1, 8, 100):
                    assert 1 <= p.kvp_decode_splits(3, 32, 8, n_q, d, n, varlen) <= 4096


def test_ranges(p):
    good = dict(o=P, pre=P, r=NONE, B=1, N=4, n=2, causal=1, stream=NONE)
    f = p.lib().vfa_row_ranges
    assert call(f, good) == INVALID
    assert call(f, good, B=0) == OK and call(f, good, N=0) == OK
    for bad in (dict(B=-1), dict(N=-1), dict(n=-1), dict(causal=2), dict(causal=-1), dict(o=ODD), dict(pre=ODD), dict(r=FOUR)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    assert call(f, good, o=NONE, r=P) == INVALID
    assert call(f, good, r=P, B=70000) == UNSUPPORTED and call(f, good, r=P, n=2 ** 31 - 1) == UNSUPPORTED and call(f, good, r=P, B=60000, N=1 << 20) == UNSUPPORTED


def test_masked(p):
    good = dict(Q=P, K=P, V=P, O=NONE, LSE=NONE, B=1, Hq=4, Hkv=2, N=4, d=64, causal=1, ranges=NONE, scale=0.0, cap=0.0, slopes=NONE, stream=NONE)
    f = p.lib().vfa_masked_attn_fwd
    assert call(f, good) == INVALID
    assert call(f, good, B=0) == OK and call(f, good, N=0) == OK
    for bad in (dict(B=-1), dict(N=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=5), dict(d=0), dict(causal=2), dict(scale=float("nan")), dict(cap=-0.5), dict(cap=float("nan")),
                dict(cap=2000.0), dict(ranges=FOUR), dict(slopes=ODD), dict(LSE=ODD)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    for d in (32, 96, 256):
        assert call(f, good, B=0, d=d) == UNSUPPORTED
    for bad in (dict(Q=NONE), dict(K=NONE), dict(V=NONE), dict(Q=FOUR), dict(K=ODD), dict(V=ODD), dict(O=FOUR)):
        assert call(f, good, **{"O": P, **bad}) == INVALID, bad
    for bad in (dict(N=1 << 25), dict(B=1 << 20, N=1 << 15), dict(B=1 << 24, Hq=1 << 10)):
        assert call(f, good, O=P, **bad) == UNSUPPORTED, bad


def test_scales_out_of_range(p):
    decode = dict(Q=P, KP=P, VP=P, table=P, O=NONE, LSE=NONE, B=0, Hq=4, Hkv=2, n_pages=9, page=16, M=8, n_q=1, d=64, lens=NONE, n_keys=4, ns=1, scale=0.0, cap=0.0,
                  slopes=NONE, ws=NONE, wsb=0, stream=NONE)
    prompt = dict(Q=P, K=P, V=P, O=NONE, LSE=NONE, B=0, Hq=4, Hkv=2, N=4, d=64, causal=1, ranges=NONE, scale=0.0, cap=0.0, slopes=NONE, stream=NONE)
    for f, good in ((p.lib().vfa_kvp_decode_fwd, decode), (p.lib().vfa_masked_attn_fwd, prompt)):
        for scale in (2.0 ** -65, 1e-40, 2.0 ** 17, 2.0 ** 64, 3e38):
            assert call(f, good, scale=scale) == INVALID, scale
        for scale in (2.0 ** -64, 2.0 ** 16, -1.0, -3e38):
            assert call(f, good, scale=scale) == OK, scale


def test_numbers_past_the_range_of_their_type(p):
    """No sequences, so that nothing is launched: a number that its C type does not hold is refused, and not taken by its low bits."""
    n = p._ns()
    append = lambda old, new: n.vfa_kvp_append(None, None, 16, 16, 16, 0, 2, 9, 16, 8, 4, 64, 8, 8, 8, 8, 8, 8, None, None, old, new, 0)
    assert append(0, 4) == OK and append(2 ** 32, 2 ** 32 + 4) == INVALID and append(0, 2 ** 32 + 4) == INVALID
    ranges = lambda N: n.vfa_row_ranges(16, None, 16, 0, N, 2, 1, 0)
    assert ranges(4) == OK and ranges(2 ** 32 + 4) == INVALID
    assert p.kvp_decode_splits(1, 4, 2, 1, 64, 2 ** 32 + 100000) == 1


# ---- what the native module looks up on tensors ------------------------------------------------------------------------------------

def pages(P=9, H=2, S=16, d=64, B=3, M=8):
    return [Fake((P, H, S, d), BF), Fake((P, H, S, d), BF), Fake((B, M), I32)]


def spoiled(make, i):
    """Every way in which one tensor of a call is not what it has to be."""
    for change in (dict(dtype="int8"), dict(device=1), dict(device=-1), dict(c=False), dict(shape=(2, 3, 4, 5, 6)), dict(shape=tuple(x + 1 for x in make()[i].shape))):
        t = make()
        for k, v in change.items():
            setattr(t[i], k, v)
        yield change, t


def test_tensors_of_append(p):
    n = p._ns()
    make = lambda: [*pages(), Fake((3, 2, 5, 64), BF), Fake((3, 2, 5, 64), BF)]
    go = lambda KP, VP, t, K, V, old=1, new=2: n.check_kvp_append(K, V, KP, VP, t, old, new, BF, I32)
    assert go(*make()) == (0, 3, 2, 9, 16, 8, 5, 64, 640, 320, 64, 640, 320, 64, None, None, 1, 2)
    a, b = Fake((3,), I32), Fake((3,), I32)
    assert go(*make(), a, b)[-4:] == (a, b, 0, 0)
    for i in range(5):
        for change, t in spoiled(make, i):
            if i >= 3 and change == dict(c=False):
                continue  # (rows may have strides)
            with pytest.raises(ValueError):
                go(*t)
    for old, new in ((a, 3), (3, b), (Fake((2,), I32), b), (a, Fake((3,), "int64")), (a, Fake((3,), I32, device=1))):
        with pytest.raises(ValueError):
            go(*make(), old, new)
    t = make()
    t[3].s = (640, 320, 64, 2)
    with pytest.raises(ValueError):
        go(*t)


def test_tensors_of_decode(p):
    n = p._ns()
    make = lambda: [*pages(), Fake((3, 4, 2, 64), BF), Fake((4,), F32)]
    go = lambda KP, VP, t, q, s, lens=7: n.check_kvp_decode(q, KP, VP, t, lens, s, BF, F32, I32)
    assert go(*make()) == (0, 3, 4, 2, 9, 16, 8, 2, 64, None, 7)
    t = make()
    t[3].shape = (3, 4, 64)
    assert go(*t) == (0, 3, 4, 2, 9, 16, 8, 1, 64, None, 7)
    assert n.check_kvp_decode(make()[3], *pages(), 7, None, BF, F32, I32)[:4] == (0, 3, 4, 2)
    for i in range(5):
        for change, t in spoiled(make, i):
            with pytest.raises(ValueError):
                go(*t)
    with pytest.raises(ValueError):
        go(*make(), Fake((2,), I32))


def test_tensors_of_ranges_and_masked(p):
    n = p._ns()
    make = lambda: [Fake((3, 6), I32), Fake((3, 5), I32)]
    go = lambda o, pre: n.check_row_ranges(o, pre, I32)
    assert go(*make()) == (0, 3, 5) and go(make()[0], None) == (0, 3, 5) and go(Fake((3, 1), I32), None) == (0, 3, 0)
    for i in range(2):
        for change, t in spoiled(make, i):
            with pytest.raises(ValueError):
                go(*t)
    with pytest.raises(ValueError):
        go(Fake((3, 0), I32), None)
    make = lambda: [Fake((3, 4, 10, 64), BF), Fake((3, 2, 10, 64), BF), Fake((3, 2, 10, 64), BF), Fake((3, 10, 2), I32), Fake((4,), F32)]
    go = lambda Q, K, V, r, s: n.check_masked_attn(Q, K, V, r, s, BF, F32, I32)
    assert go(*make()) == (0, 3, 4, 2, 10, 64) and go(*make()[:3], None, None) == (0, 3, 4, 2, 10, 64)
    for i in range(5):
        for change, t in spoiled(make, i):
            with pytest.raises(ValueError):
                go(*t)


def test_wrappers_refuse(p, monkeypatch):
    """Tensors of another GPU than the current one, and wrong outputs."""
    import torch
    host = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    for f in (lambda: p.masked_attn_fwd(host, host, host), lambda: p.kvp_append(host, host, (host, host), torch.zeros((1, 2), dtype=torch.int32), 0, 1),
              lambda: p.kvp_decode_fwd(host, (host, host), torch.zeros((1, 2), dtype=torch.int32), 1), lambda: p.row_ranges(torch.zeros((1, 2), dtype=torch.int32), 4)):
        with pytest.raises(ValueError):
            f()
    monkeypatch.setattr(p, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current GPU"):
        p.row_ranges(Fake((1, 2), torch.int32), 4)
