"""What the native module looks up on the tensors of the serving operators, and what it refuses.  CPU only: objects that only look like tensors."""
import os
import sys

import pytest

from paper_2604_12798_amd import build


@pytest.fixture(scope="module")
def n():
    import paper_2604_12798_amd as p
    if not os.path.exists(p.LIB_PATH) or not os.path.exists(build.BINDING):
        build.build_lib()
    return p._n()


class Fake:
    def __init__(self, shape, dtype, device=0, contiguous=True, stride=None):
        self.shape, self.dtype, self.device, self.c = shape, dtype, device, contiguous
        if stride is None:
            stride, size = [], 1
            for x in reversed(shape):
                stride.insert(0, size)
                size *= x
        self.s = tuple(stride)

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.c

    def stride(self):
        return self.s

    def dim(self):
        return len(self.shape)


U8, BF, F32, I32 = "uint8", "bfloat16", "float32", "int32"


def check_cache8(n, *args, lens=7):
    return n.check_cache8(*args[:4], lens, *args[4:], I32)


def check_append(n, K, V, c, old=1, new=2):
    return n.check_kv8_append(K, V, *c, old, new, BF, U8, I32)


def check_decode(n, q, c, lens=9):
    return n.check_kv8_decode(q, *c, lens, BF, U8, I32)


def check_rope(n, q, k, v, qw=None, kw=None, cs=None, first=3):
    return n.check_norm_rope(q, k, v, qw, kw, cs, first, BF, F32, I32)


def cache(B=2, H=3, T=4, s=2, **kw):
    shapes = [(B, H, T, s, 64, 64), (B, H, T, 64 * s, 64), (B, H, T), (B, H, T)]
    return [Fake(x, U8, **kw) for x in shapes]


def test_cache(n):
    assert check_cache8(n, *cache(), U8) == (0, 2, 3, 256, 128, None, 7)
    assert check_cache8(n, *cache(s=1, device=5), U8) == (5, 2, 3, 256, 64, None, 7)
    assert check_cache8(n, *cache(B=0), U8) == (0, 0, 3, 256, 128, None, 7)
    lens = Fake((2,), I32)
    assert check_cache8(n, *cache(), U8, lens=lens) == (0, 2, 3, 256, 128, lens, 0)
    for i in range(4):
        for change in (dict(dtype="int8"), dict(device=1), dict(device=-1), dict(c=False), dict(shape=(2, 3)), dict(shape=cache()[i].shape[:-1] + (63,)),
                       dict(shape=(1,) + cache()[i].shape[1:])):
            c = cache()
            for k, v in change.items():
                setattr(c[i], k, v)
            with pytest.raises(ValueError):
                check_cache8(n, *c, U8)
    with pytest.raises(ValueError):
        check_cache8(n, *cache(device=-1), U8)  # on the host
    for bad in (lambda: n.check_cache8(*cache()), lambda: n.check_kv8_append(1), lambda: n.check_kv8_decode(1), lambda: n.check_norm_rope(1),
                lambda: n.check_tensor(1, 2)):
        with pytest.raises(TypeError):
            bad()


def test_append(n):
    K = Fake((2, 3, 5, 128), BF, stride=(1000, 128, 2000, 1))
    V = Fake((2, 3, 5, 128), BF)
    assert check_append(n, K, V, cache()) == (0, 2, 3, 256, 5, 128, 1000, 128, 2000, 3 * 5 * 128, 5 * 128, 128, None, None, 1, 2)
    for t in (Fake((2, 3, 5, 64), BF), Fake((2, 3, 6, 128), BF), Fake((2, 2, 5, 128), BF), Fake((1, 3, 5, 128), BF), Fake((2, 3, 5, 128), U8),
              Fake((2, 3, 5, 128), BF, device=1), Fake((2, 3, 5, 128), BF, stride=(1, 1, 1, 2)), Fake((3, 5, 128), BF)):
        for pair in ((t, V), (K, t)):
            with pytest.raises(ValueError):
                check_append(n, *pair, cache())


def test_decode(n):
    assert check_decode(n, Fake((2, 6, 4, 128), BF), cache()) == (0, 2, 6, 3, 256, 4, 128, None, 9)
    assert check_decode(n, Fake((2, 6, 128), BF), cache()) == (0, 2, 6, 3, 256, 1, 128, None, 9)
    for q in (Fake((2, 6, 64), BF), Fake((1, 6, 128), BF), Fake((2, 6, 128), U8), Fake((2, 6, 128), BF, contiguous=False), Fake((2, 6, 128), BF, device=1),
              Fake((2, 128), BF), Fake((2, 6, 1, 1, 128), BF)):
        with pytest.raises(ValueError):
            check_decode(n, q, cache())


def test_norm_rope(n):
    q = Fake((2, 7, 8, 64), BF, stride=(10000, 1000, 64, 1))
    k, v = Fake((2, 7, 2, 64), BF), Fake((2, 7, 2, 64), BF, stride=(9, 8, 7, 1))
    assert check_rope(n, q, k, v) == (0, 2, 7, 8, 2, 64, 10000, 1000, 64, 7 * 128, 128, 64, 9, 8, 7, 0, 0, None, 3)
    assert check_rope(n, q, k, None)[-7:-4] == (0, 0, 0)
    for t in (Fake((2, 7, 2, 128), BF), Fake((2, 6, 2, 64), BF), Fake((1, 7, 2, 64), BF), Fake((2, 7, 2, 64), U8), Fake((2, 7, 2, 64), BF, device=2),
              Fake((2, 7, 2, 64), BF, stride=(1, 1, 1, 3)), Fake((7, 2, 64), BF)):
        for args in ((t, k, v), (q, t, v), (q, k, t)):
            with pytest.raises(ValueError):
                check_rope(n, *args)
    with pytest.raises(ValueError):
        check_rope(n, q, k, Fake((2, 7, 1, 64), BF))
    w, cs, first = Fake((64,), BF), Fake((50, 32), F32), Fake((2,), I32)
    assert check_rope(n, q, k, v, w, w, cs, first)[-4:] == (50, 32, first, 0)
    for i, bads in enumerate(((Fake((63,), BF), Fake((64,), F32), Fake((1, 64), BF), Fake((64,), BF, device=1)),
                              (Fake((64,), BF, contiguous=False), Fake((128,), BF)),
                              (Fake((50, 32), BF), Fake((50,), F32), Fake((50, 32), F32, contiguous=False), Fake((50, 32), F32, device=-1)),
                              (Fake((3,), I32), Fake((2,), "int64"), Fake((2, 1), I32), Fake((2,), I32, device=1)))):
        for bad in bads:
            args = [w, w, cs, first]
            args[i] = bad
            with pytest.raises(ValueError):
                check_rope(n, q, k, v, *args)


def test_lengths(n):
    """Numbers as Python takes them for whole ones; anything else is an error of its own."""
    K, c, lens = Fake((2, 3, 5, 128), BF), cache(), Fake((2,), I32)
    assert check_append(n, K, K, c, True, 2 ** 40)[-4:] == (None, None, 1, 2 ** 40)
    assert check_append(n, K, K, c, lens, lens)[-4:] == (lens, lens, 0, 0)
    for pair in ((lens, 3), (3, lens), (Fake((2,), I32, contiguous=False), lens), (lens, Fake((1,), I32))):
        with pytest.raises(ValueError):
            check_append(n, K, K, c, *pair)
    for bad in (None, [1], object()):
        with pytest.raises(TypeError):
            check_decode(n, Fake((2, 6, 128), BF), c, bad)


def test_strides_of_one_entry(n):
    """An axis of one entry may have any stride."""
    x = Fake((1, 1, 1, 64), BF, stride=(3, 5, 7, 1))
    assert check_rope(n, x, x, x)[6:15] == (0,) * 9
    assert check_append(n, Fake((1, 3, 1, 128), BF, stride=(1, 128, 1, 1)), Fake((1, 3, 1, 128), BF), cache(B=1))[6:12] == (0, 128, 0, 0, 128, 0)


def test_tensor(n):
    t = Fake((3, 4), BF)
    assert n.check_tensor(t, BF, 0, 3, 4) is True
    for bad in ((t, U8, 0, 3, 4), (t, BF, 1, 3, 4), (t, BF, 0, 3, 5), (t, BF, 0, 12), (t, BF, 0, 3, 4, 1), (Fake((3, 4), BF, contiguous=False), BF, 0, 3, 4),
                (Fake((3, 4), BF, device=-1), BF, 0, 3, 4)):
        assert n.check_tensor(*bad) is False
    with pytest.raises(AttributeError):
        n.check_tensor(1, BF, 0, 3)


def test_errors_pass_through_and_nothing_is_kept(n):
    class Bad(Fake):
        def get_device(self):
            raise KeyError("mine")
    with pytest.raises(KeyError):
        n.check_tensor(Bad((3,), BF), BF, 0, 3)
    with pytest.raises(KeyError):
        check_decode(n, Bad((2, 6, 128), BF), cache())
    good = [Fake((2, 6, 128), BF)] + cache() + [Fake((2,), I32)]
    bad = Fake((2, 6, 64), BF)
    before = [sys.getrefcount(x) for x in good + [bad]]
    for _ in range(100):
        check_decode(n, good[0], good[1:5], good[5])
        with pytest.raises(ValueError):
            check_decode(n, bad, good[1:5])
    after = [sys.getrefcount(x) for x in good + [bad]]
    assert all(abs(a - b) <= 2 for a, b in zip(after, before))
