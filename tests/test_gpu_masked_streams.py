"""The paged cache's and masked attention's wrappers on another stream than the current one, with memory of their own, while the current stream allocates and writes: before
the call runs, and in memory that it freed with work of its own still to come."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as pkg
    pkg.lib()
    return pkg


def rnd(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def make(vfa, name):
    """The call, and the bytes of what it allocates."""
    B, Hq, H, N, d = 2, 8, 2, 512, 128
    Q, K, V = rnd((B, Hq, N, d), 1), rnd((B, H, N, d), 2), rnd((B, H, N, d), 3)
    cache = vfa.kvp_cache(70, H, 16, d)
    table = torch.arange(64, dtype=torch.int32, device="cuda").reshape(2, 32)
    vfa.kvp_append(K, V, cache, table, 0, N)
    lens = torch.tensor([512, 130], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([[0, 100, 512], [5, 300, 400]], dtype=torch.int32, device="cuda")
    ranges = vfa.row_ranges(offsets, N)
    q = Q[:, :, :2].contiguous()
    out, lse, ws = Q.numel() * 2, B * Hq * N * 4, vfa.kvp_decode_workspace_bytes(B, Hq, 2, d, 5)
    o, l = torch.empty_like(q), torch.empty((B, Hq, 2), device="cuda")
    return {
        "kvp_decode_fwd": (lambda **s: vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=5, **s), (q.numel() * 2, B * Hq * 2 * 4, ws)),
        "kvp_decode_fwd, outputs given": (lambda **s: vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=5, out=o, lse=l, **s), (ws,)),
        "kvp_decode_fwd, no LSE": (lambda **s: vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=5, want_lse=False, **s), (q.numel() * 2, ws)),
        "row_ranges": (lambda **s: (vfa.row_ranges(offsets, N, **s),), (B * N * 8,)),
        "masked_attn_fwd": (lambda **s: vfa.masked_attn_fwd(Q, K, V, ranges=ranges, score_cap=30.0, **s), (out, lse)),
        "masked_attn_fwd, no LSE": (lambda **s: vfa.masked_attn_fwd(Q, K, V, ranges=ranges, want_lse=False, **s), (out,)),
    }[name]


@pytest.mark.parametrize("name", ["kvp_decode_fwd", "kvp_decode_fwd, outputs given", "kvp_decode_fwd, no LSE", "row_ranges", "masked_attn_fwd", "masked_attn_fwd, no LSE"])
def test_the_current_stream_goes_on(vfa, name):
    call, sizes = make(vfa, name)
    want = [t.clone() for t in call() if t is not None]
    a = torch.ones((4096, 4096), dtype=torch.bfloat16, device="cuda")
    b = torch.empty_like(a)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def busy():
        for _ in range(20):
            torch.mm(a, a, out=b)

    for turn in range(3):
        # the call waits on its stream; what the current one allocates and writes meanwhile is not the call's
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            busy()
        got = call(stream=s)
        junk = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip([t for t in got if t is not None], want)), turn
        # memory that the current stream freed and has still to write
        s.wait_stream(torch.cuda.current_stream())
        busy()
        for t in junk:
            t.fill_(0xFF)
        del junk, t, got
        got = call(stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip([t for t in got if t is not None], want)), turn
        del got
