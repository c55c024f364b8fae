"""The paged cache's and masked attention's wrappers with memory of their own, called for another stream than the current one.  CPU only."""
import pytest

from test_wrapper_streams import BF, CURRENT, F32, I32, OTHER, U8, Tensor, p, world  # noqa: F401


def calls(p, w):
    """Each wrapper that allocates something: (call with something of its own to allocate, how many, call with everything given or None)."""
    t = lambda shape, dtype=BF: Tensor(w, shape, dtype)
    Q, K = t((1, 4, 128, 128)), t((1, 2, 128, 128))
    q, lens, table = t((1, 4, 3, 128)), t((1,), I32), t((1, 8), I32)
    cache = (t((9, 2, 16, 128)), t((9, 2, 16, 128)))
    out, lse, ws = dict(out=t(q.shape)), dict(lse=t(q.shape[:3], F32)), dict(workspace=t((1 << 20,), U8))
    offsets, ranges = t((1, 4), I32), t((1, 50, 2), I32)
    decode = lambda **kw: p.kvp_decode_fwd(q, cache, table, lens, n_splits=3, **kw)
    prompt = lambda **kw: p.masked_attn_fwd(Q, K, K, **kw)
    O, L = dict(out=t(Q.shape)), dict(lse=t(Q.shape[:3], F32))
    return {
        "kvp_decode_fwd": (lambda **s: decode(**s), 3, lambda **s: decode(**out, **lse, **ws, **s)),
        "kvp_decode_fwd, one range": (lambda **s: p.kvp_decode_fwd(q, cache, table, 100, n_splits=1, **s), 2, None),
        "kvp_decode_fwd, outputs given": (lambda **s: decode(**out, **lse, **s), 1, None),
        "kvp_decode_fwd, workspace given": (lambda **s: decode(**ws, **s), 2, None),
        "kvp_decode_fwd, but for the LSE": (lambda **s: decode(**out, **ws, **s), 1, None),
        "kvp_decode_fwd, no LSE": (lambda **s: decode(want_lse=False, **s), 2, lambda **s: decode(want_lse=False, **out, **ws, **s)),
        "row_ranges": (lambda **s: p.row_ranges(offsets, 50, **s), 1, lambda **s: p.row_ranges(offsets, 50, out=ranges, **s)),
        "masked_attn_fwd": (lambda **s: prompt(**s), 2, lambda **s: prompt(**O, **L, **s)),
        "masked_attn_fwd, but for the LSE": (lambda **s: prompt(**O, **s), 1, None),
        "masked_attn_fwd, but for the output": (lambda **s: prompt(**L, **s), 1, None),
        "masked_attn_fwd, no LSE": (lambda **s: prompt(want_lse=False, **s), 1, lambda **s: prompt(want_lse=False, **O, **s)),
    }


@pytest.mark.parametrize("name", list(calls(None, None)))
def test_memory_for_another_stream_is_that_streams(p, world, name):  # noqa: F811
    w = world
    something, n, everything = calls(p, w)[name]
    out = something(stream=OTHER)
    assert len(w.made) == n and w.launches and all(h == OTHER.cuda_stream for _, h in w.launches)
    assert all(t.made_on is OTHER for t in w.made) and w.now is CURRENT
    out = out if isinstance(out, tuple) else (out,)
    for t in w.made:
        assert t.recorded == ([CURRENT] if any(t is o for o in out) else [])
    for same in (dict(), dict(stream=None), dict(stream=CURRENT)):
        w.made, w.launches, w.entered = [], [], 0
        something(**same)
        assert len(w.made) == n and all(t.made_on is CURRENT and not t.recorded for t in w.made)
        assert all(h == CURRENT.cuda_stream for _, h in w.launches) and w.entered == 0
    if everything is not None:
        w.made, w.launches, w.entered = [], [], 0
        everything(stream=OTHER)
        assert not w.made and w.launches and all(h == OTHER.cuda_stream for _, h in w.launches) and w.entered == 0
