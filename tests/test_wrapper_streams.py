"""Memory that the Python wrappers allocate for a call on another stream than the current one.  CPU only: objects that only look like tensors and streams."""
import contextlib
import os

import pytest
import torch

from paper_2604_12798_amd import build


@pytest.fixture(scope="module")
def p():
    import paper_2604_12798_amd as pkg
    if not os.path.exists(pkg.LIB_PATH) or not os.path.exists(build.BINDING):
        build.build_lib()
    pkg._ns()
    return pkg


BF, U8, I32, F32 = torch.bfloat16, torch.uint8, torch.int32, torch.float32


class Stream:
    device_index = 0

    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, OTHER = Stream(11), Stream(22)


class World:
    """The current stream, what was allocated on which one, and the launches."""

    def __init__(self):
        self.now, self.made, self.launches, self.entered = CURRENT, [], [], 0

    @contextlib.contextmanager
    def stream(self, s):
        before, self.now = self.now, s
        self.entered += 1
        try:
            yield
        finally:
            self.now = before

    def empty(self, shape, dtype=None, device=None):
        t = Tensor(self, (shape,) if isinstance(shape, int) else shape, dtype)
        t.made_on = self.now
        self.made.append(t)
        return t


class Tensor:
    is_cuda, device, made_on = True, "cuda:0", None

    def __init__(self, world, shape, dtype):
        self.world, self.shape, self.dtype, self.recorded = world, tuple(shape), dtype, []

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def stride(self):
        out, size = [], 1
        for x in reversed(self.shape):
            out.insert(0, size)
            size *= x
        return tuple(out)

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def element_size(self):
        return {BF: 2, U8: 1, I32: 4, F32: 4}[self.dtype]

    def new_empty(self, shape, dtype=None):
        return self.world.empty(shape, dtype or self.dtype)

    def record_stream(self, s):
        self.recorded.append(s)


class Native:
    def __init__(self, world, native):
        self.world, self.native = world, native

    def __getattr__(self, name):
        if not name.endswith("_t"):
            return getattr(self.native, name)

        def launch(*args):
            self.world.launches.append((name, args[-1]))
            return 0
        return launch


@pytest.fixture
def world(p, monkeypatch):
    w = World()
    monkeypatch.setattr(p, "_native", Native(w, p._ns()))
    monkeypatch.setattr(p, "_empty_like", lambda t: w.empty(t.shape, t.dtype))
    monkeypatch.setattr(p, "_current_device", lambda: 0)
    monkeypatch.setattr(p, "_current_stream", lambda device: w.now.cuda_stream)
    monkeypatch.setattr(torch, "empty", w.empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: w.empty(t.shape, t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", w.stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: w.now)
    return w


def calls(p, w):
    """Each wrapper that allocates something: (call with nothing given, call with everything given or None)."""
    t = lambda shape, dtype=BF: Tensor(w, shape, dtype)
    Q, K = t((1, 4, 128, 128)), t((1, 2, 128, 128))
    kw = dict(out=t(Q.shape), lse=t(Q.shape[:3], F32))
    ws = dict(workspace=t((1 << 20,), U8))
    mask = dict(skip_mask=t((1, 4, 1, 2), U8))
    q, lens = t((1, 4, 128)), t((1,), I32)
    qkw = dict(out=t(q.shape), lse=t((1, 4), F32), **ws)
    Q8, K8, V8, Q4, K4, QS, KS = t(Q.shape, U8), t(K.shape, U8), t((1, 2, 2, 128, 64), U8), t((1, 4, 128, 64), U8), t((1, 2, 128, 64), U8), t((1, 4, 128, 4), U8), t((1, 2, 128, 4), U8)
    f8, f4 = dict(descale_q=1, descale_k=1, descale_v=1), dict(descale_v=1)
    cache = (t((1, 2, 2, 2, 64, 64), U8), t((1, 2, 2, 128, 64), U8), t((1, 2, 2), U8), t((1, 2, 2), U8))
    x, y = t((1, 3, 4, 128)), t((1, 3, 2, 128))
    rope = dict(out=(t((1, 4, 3, 128)), t((1, 2, 3, 128)), t((1, 2, 3, 128))))
    return {
        "kblock_summary": (lambda **s: p.kblock_summary(K, **s), lambda **s: p.kblock_summary(K, out=t((1, 2, 2, 128)), **s)),
        "kblock_summary_mode": (lambda **s: p.kblock_summary(K, repr_mode=2, **s), None),
        "fa_baseline_fwd": (lambda **s: p.fa_baseline_fwd(Q, K, K, **s), lambda **s: p.fa_baseline_fwd(Q, K, K, **kw, **s)),
        "fa_lazy_rescale_fwd": (lambda **s: p.fa_lazy_rescale_fwd(Q, K, K, **s), lambda **s: p.fa_lazy_rescale_fwd(Q, K, K, **kw, **s)),
        "fa_lazy_rescale_softexp_fwd": (lambda **s: p.fa_lazy_rescale_softexp_fwd(Q, K, K, **s), lambda **s: p.fa_lazy_rescale_softexp_fwd(Q, K, K, **kw, **s)),
        "vfa_attn_fwd": (lambda **s: p.vfa_attn_fwd(Q, K, K, **s), lambda **s: p.vfa_attn_fwd(Q, K, K, **kw, **ws, **s)),
        "vfa_attn_fwd, outputs given": (lambda **s: p.vfa_attn_fwd(Q, K, K, **kw, **s), None),
        "vsa_attn_fwd": (lambda **s: p.vsa_attn_fwd(Q, K, K, **s), lambda **s: p.vsa_attn_fwd(Q, K, K, **kw, **ws, **mask, **s)),
        "vsa_attn_fwd, but for the mask": (lambda **s: p.vsa_attn_fwd(Q, K, K, **kw, **ws, **s), None),
        "vfa_variant_fwd": (lambda **s: p.vfa_variant_fwd(Q, K, K, skip_threshold_nats=1.0, **s),
                            lambda **s: p.vfa_variant_fwd(Q, K, K, skip_threshold_nats=1.0, **kw, **ws, **mask, **s)),
        "vfa_variant_fwd, summaries of queries": (lambda **s: p.vfa_variant_fwd(Q, K, K, q_repr_mode=1, **kw, **s), None),
        "vfa_variant_fwd, but for the mask": (lambda **s: p.vfa_variant_fwd(Q, K, K, skip_threshold_nats=1.0, **kw, **ws, **s), None),
        "decode_fwd": (lambda **s: p.decode_fwd(q, K, K, 100, **s), lambda **s: p.decode_fwd(q, K, K, 100, **qkw, **s)),
        "decode_varlen_fwd": (lambda **s: p.decode_varlen_fwd(q, K, K, lens, **s), lambda **s: p.decode_varlen_fwd(q, K, K, lens, **qkw, **s)),
        "fp8_quantize": (lambda **s: p.fp8_quantize(Q, 1.0, **s), None),
        "fp8_pack_v": (lambda **s: p.fp8_pack_v(K, 1.0, **s), None),
        "fp8_attn_fwd": (lambda **s: p.fp8_attn_fwd(Q8, K8, V8, **f8, **s), lambda **s: p.fp8_attn_fwd(Q8, K8, V8, **f8, **kw, **ws, **s)),
        "fp8_attn_fwd, no exponential": (lambda **s: p.fp8_attn_fwd(Q8, K8, V8, noexp=True, **f8, **s), None),
        "mxfp4_quantize": (lambda **s: p.mxfp4_quantize(Q, **s), None),
        "mxfp4_attn_fwd": (lambda **s: p.mxfp4_attn_fwd(Q4, QS, K4, KS, V8, **f4, **s), lambda **s: p.mxfp4_attn_fwd(Q4, QS, K4, KS, V8, **f4, **kw, **ws, **s)),
        "qk_norm_rope_fwd": (lambda **s: p.qk_norm_rope_fwd(x, y, y, **s), lambda **s: p.qk_norm_rope_fwd(x, y, y, **rope, **s)),
        "kv8_read": (lambda **s: p.kv8_read(cache, 100, **s), lambda **s: p.kv8_read(cache, 100, out=(t((1, 2, 100, 128)), t((1, 2, 100, 128))), **s)),
        "kv8_decode_fwd": (lambda **s: p.kv8_decode_fwd(q, cache, 100, n_splits=3, **s), lambda **s: p.kv8_decode_fwd(q, cache, lens, n_splits=3, **qkw, **s)),
        "kv8_decode_fwd, outputs given": (lambda **s: p.kv8_decode_fwd(q, cache, lens, n_splits=3, out=t(q.shape), lse=t((1, 4), F32), **s), None),
        "kv8_decode_fwd, no LSE": (lambda **s: p.kv8_decode_fwd(q, cache, lens, n_splits=3, want_lse=False, **s),
                                   lambda **s: p.kv8_decode_fwd(q, cache, lens, n_splits=3, out=t(q.shape), want_lse=False, **ws, **s)),
    }


NAMES = list(calls(None, None))


@pytest.mark.parametrize("name", NAMES)
def test_memory_for_another_stream_is_that_streams(p, world, name):
    """What a wrapper allocates belongs to the stream that the kernels run on: freed or not, nobody else's work can be in it before or meanwhile.  An output
    is the caller's, who uses it on the stream that was current: it is not given to others before that stream is through with it."""
    w = world
    nothing, everything = calls(p, w)[name]
    out = nothing(stream=OTHER)
    assert w.made and w.launches and all(h == OTHER.cuda_stream for _, h in w.launches)
    assert all(t.made_on is OTHER for t in w.made)
    out = out if isinstance(out, tuple) else (out,)
    for t in w.made:
        if any(t is o for o in out):
            assert t.recorded == [CURRENT]
    assert w.now is CURRENT
    for same in (dict(), dict(stream=None), dict(stream=CURRENT)):
        w.made, w.launches, w.entered = [], [], 0
        nothing(**same)
        assert all(t.made_on is CURRENT and not t.recorded for t in w.made)
        assert w.made and all(h == CURRENT.cuda_stream for _, h in w.launches) and w.entered == 0
    if everything is not None:
        w.made, w.launches, w.entered = [], [], 0
        everything(stream=OTHER)
        assert not w.made and w.launches and all(h == OTHER.cuda_stream for _, h in w.launches) and w.entered == 0
