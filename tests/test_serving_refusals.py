"""What the serving operators refuse, before anything is launched.  CPU only."""
import ctypes
import os

import pytest

OK, INVALID, UNSUPPORTED = 0, -1, -2
P, ODD, NONE = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002), ctypes.c_void_p(0)  # never dereferenced


@pytest.fixture(scope="module")
def L():
    import paper_2604_12798_amd as p
    if not os.path.exists(p.LIB_PATH):
        from paper_2604_12798_amd import build
        build.build_lib()
    return p.lib()


def call(f, good, **changed):
    assert set(changed) <= set(good), changed
    return f(*{**good, **changed}.values())


def test_norm_rope(L):
    good = dict(Xq=P, Xk=P, Xv=P, Q=P, K=P, V=P, B=1, N=4, Hq=4, Hkv=2, d=128, qb=1, qn=1, qh=8, kb=8, kn=8, kh=8, vb=8, vn=8, vh=8, norm=1,
                qw=P, kw=P, eps=1e-6, cs=P, n_pos=8, rot=64, inter=0, fp=NONE, first=0, stream=NONE)
    f = L.vfa_qk_norm_rope_fwd   # (the strides of `good` are refused, so that no variation below can get as far as a launch)
    assert call(f, good) == INVALID
    assert call(f, good, B=0) == OK and call(f, good, N=0) == OK
    for bad in (dict(B=-1), dict(N=-1), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(rot=-16), dict(rot=8), dict(rot=144), dict(norm=2), dict(inter=-1),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(cs=NONE), dict(cs=ODD), dict(n_pos=0), dict(fp=ODD), dict(norm=0)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    for d in (96, 32, 256):
        assert call(f, good, B=0, d=d) == UNSUPPORTED
    assert call(f, good, B=0, rot=0, cs=NONE, n_pos=0) == OK
    assert call(f, good, B=0, norm=0, qw=NONE, kw=NONE) == OK
    for bad in (dict(Xq=NONE), dict(Xk=NONE), dict(Xv=NONE), dict(Q=NONE), dict(K=NONE), dict(V=NONE), dict(Xq=ODD), dict(V=ODD), dict(qw=ODD)):
        assert call(f, good, **bad) == INVALID, bad
    flat = dict(qb=8, qn=8, qh=8)
    for name in ("kb", "kn", "kh", "vb", "vn", "vh"):
        assert call(f, good, **{**flat, name: 4}) == INVALID
    assert call(f, good, **flat, B=1 << 16, N=1 << 16) == UNSUPPORTED
    assert call(f, good, **flat, N=1 << 20, Hq=1 << 20) == UNSUPPORTED


def test_append(L):
    good = dict(K=P, V=P, K8=P, V8=P, KS=P, VS=P, B=1, Hkv=2, cap=128, n_in=4, d=64, kb=1, kh=8, kn=8, vb=8, vh=8, vn=8, ol=NONE, nl=NONE, old=0, new=4,
                stream=NONE)
    f = L.vfa_kv8_append
    assert call(f, good) == INVALID  # (a stride of 1)
    assert call(f, good, B=0) == OK and call(f, good, n_in=0, new=0) == OK and call(f, good, old=4) == OK
    assert call(f, good, cap=0, new=0) == OK
    for bad in (dict(B=-1), dict(Hkv=0), dict(cap=-64), dict(n_in=-1), dict(d=-1), dict(old=-1), dict(old=5), dict(new=129), dict(new=5), dict(ol=P), dict(nl=P),
                dict(ol=ODD, nl=P), dict(ol=P, nl=ODD)):
        assert call(f, good, **{"B": 0, **bad}) == INVALID, bad
    for bad in (dict(d=96), dict(cap=100), dict(cap=1)):
        assert call(f, good, **bad) == UNSUPPORTED, bad
    ok = dict(kb=8)
    for bad in (dict(K=NONE), dict(V=NONE), dict(K8=NONE), dict(V8=NONE), dict(KS=NONE), dict(VS=NONE), dict(K=ODD), dict(V=ODD), dict(K8=ODD), dict(V8=ODD),
                dict(vn=4), dict(vb=12), dict(kh=-4)):
        assert call(f, good, **{**ok, **bad}) == INVALID, bad
    assert call(f, good, **ok, B=40000) == UNSUPPORTED
    assert call(f, good, **ok, B=1, Hkv=40000) == UNSUPPORTED
    assert call(f, good, **ok, B=1000, Hkv=60, cap=1 << 20, n_in=1 << 20, new=1 << 20) == UNSUPPORTED


def test_read(L):
    good = dict(K8=P, V8=P, KS=P, VS=P, K=P, V=P, B=1, Hkv=2, cap=128, n=100, d=64, lens=NONE, length=100, stream=NONE)
    f = L.vfa_kv8_read
    assert call(f, good, B=0) == OK and call(f, good, n=0) == OK
    for bad in (dict(B=-1), dict(Hkv=0), dict(cap=-64), dict(n=-1), dict(n=129), dict(lens=ODD), dict(K=NONE), dict(V=NONE), dict(K=ODD), dict(V=ODD), dict(K8=NONE),
                dict(V8=ODD), dict(KS=NONE), dict(VS=NONE)):
        assert call(f, good, **bad) == INVALID, bad
    for bad in (dict(d=96), dict(cap=100), dict(B=40000)):
        assert call(f, good, **bad) == UNSUPPORTED, bad


def test_decode(L):
    good = dict(Q=P, K8=P, V8=P, KS=P, VS=P, O=P, LSE=P, B=1, Hq=8, Hkv=2, cap=128, n_q=1, d=64, lens=NONE, n=100, splits=2, scale=0.0, ws=P, bytes=1 << 20,
                stream=NONE)
    f = L.vfa_kv8_decode_fwd
    assert call(f, good, B=0) == OK and call(f, good, n_q=0) == OK
    for bad in (dict(B=-1), dict(Hq=0), dict(Hq=9), dict(Hkv=0), dict(cap=-64), dict(n_q=-1), dict(lens=ODD), dict(n=-1), dict(n=129), dict(splits=0), dict(splits=4097),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(Q=NONE), dict(O=NONE), dict(Q=ODD), dict(O=ODD), dict(LSE=ODD), dict(K8=NONE), dict(KS=NONE),
                dict(V8=ODD), dict(ws=NONE), dict(ws=ODD), dict(bytes=100)):
        assert call(f, good, **bad) == INVALID, bad
    for bad in (dict(d=32), dict(cap=127), dict(Hq=66), dict(B=40000), dict(Hq=66, n_q=2), dict(n_q=1 << 29), dict(n_q=1 << 24), dict(Hq=32, n_q=65536 * 2 + 1), dict(B=20000, n_q=20000), dict(Hq=1, Hkv=1, n_q=2 ** 31 - 1)):
        assert call(f, good, **bad) == UNSUPPORTED, bad
    assert L.vfa_kv8_decode_workspace_bytes(2, 8, 3, 64, 5) == (2 * 8 * 3 * 5 * 66 * 4 + 16 + 255) // 256 * 256
    assert L.vfa_kv8_decode_workspace_bytes(0, 8, 3, 64, 5) == 0 and L.vfa_kv8_decode_workspace_bytes(1, 8, 0, 64, 5) == 0
    for B, H, n in ((1, 1, 1), (1, 8, 4096), (64, 8, 100000), (1, 1, 1 << 30), (0, 1, 1), (100000, 100000, 1)):
        for d in (64, 128):
            for varlen in (0, 1):
                assert 1 <= L.vfa_kv8_decode_splits(B, 4 * H, H, 2, d, n, varlen) <= 4096
    assert L.vfa_kv8_decode_splits(1, 64, 1, 2 ** 31 - 1, 64, 2 ** 31 - 64, 1) == 1 and L.vfa_kv8_decode_splits(1, 1, 1, 2 ** 31 - 1, 64, 4096, 0) == 1
    big = 2 ** 31 - 1
    assert L.vfa_kv8_decode_splits(big, big, big, big, 64, big, 1) == 1 and L.vfa_kv8_decode_splits(65535, big, 1, big, 128, big, 0) == 1
    assert L.vfa_kv8_decode_splits(1, 0, 1, 1, 64, 4096, 0) == 1 and L.vfa_kv8_decode_splits(1, 1, 1, 0, 64, 4096, 0) == 1


def test_wrappers_refuse_tensors_that_do_not_fit():
    """On the host alone every tensor is on the wrong device."""
    import torch
    import paper_2604_12798_amd as p
    if torch.cuda.is_available():
        pytest.skip("for hosts without a GPU")
    cache = p.kv8_cache(1, 2, 100, 64, device="cpu")
    assert cache[0].shape == (1, 2, 2, 1, 64, 64) and cache[1].shape == (1, 2, 2, 64, 64)
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    for bad in (lambda: p.kv8_append(x, x, cache, 0, 3), lambda: p.kv8_read(cache, 3), lambda: p.kv8_decode_fwd(x, cache, 3), lambda: p.qk_norm_rope_fwd(x, x)):
        with pytest.raises(ValueError):
            bad()
