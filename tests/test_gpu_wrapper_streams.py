"""Calls on another stream than the current one with memory of their own, while the current stream allocates and writes: before the call runs, and in
memory that it freed with work of its own still to come."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2604_12798_amd as pkg
    pkg.lib()
    return pkg


def rnd(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def make(vfa, name):
    """The call, and the bytes of what it allocates."""
    B, Hq, H, N, d = 2, 8, 2, 512, 128
    Q, K, V = rnd((B, Hq, N, d), 1), rnd((B, H, N, d), 2), rnd((B, H, N, d), 3)
    lens = torch.tensor([512, 130], dtype=torch.int32, device="cuda")
    cache = vfa.kv8_append(K, V, vfa.kv8_cache(B, H, N, d), 0, N)
    x, y = rnd((B, N, Hq, d), 4), rnd((B, N, H, d), 5)
    q = Q[:, :, :2].contiguous()
    one, R = q[:, :, 0].contiguous(), vfa.kblock_summary(K)
    out = Q.numel() * 2
    return {
        "kv8_decode_fwd": (lambda **s: vfa.kv8_decode_fwd(q, cache, lens, n_splits=5, **s),
                           (q.numel() * 2, q.numel() * 4 // d, vfa.kv8_decode_workspace_bytes(B, Hq, 2, d, 5))),
        "kv8_read": (lambda **s: vfa.kv8_read(cache, N, seq_lens=lens, **s), (K.numel() * 2,)),
        "qk_norm_rope_fwd": (lambda **s: vfa.qk_norm_rope_fwd(x, y, y, **s), (out, K.numel() * 2)),
        "vfa_attn_fwd": (lambda **s: vfa.vfa_attn_fwd(Q, K, V, **s), (out, B * Hq * N * 4, vfa.workspace_bytes(B, H, N, d, 64))),
        "decode_fwd": (lambda **s: vfa.decode_fwd(one, K, V, 500, krepr=R, **s), (B * Hq * d * 2, B * Hq * 4, vfa.decode_workspace_bytes(B, Hq, d, 8))),
    }[name]


@pytest.mark.parametrize("name", ["kv8_decode_fwd", "kv8_read", "qk_norm_rope_fwd", "vfa_attn_fwd", "decode_fwd"])
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


def test_outputs_are_kept_until_the_current_stream_is_through(vfa):
    """An output that the caller reads on the current stream and drops is not given to the next call on the other one before that read."""
    call, _ = make(vfa, "kv8_read")
    want = call()[0].clone()
    a = torch.ones((4096, 4096), dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    copies = []
    for turn in range(4):
        s.wait_stream(torch.cuda.current_stream())
        K, V = call(stream=s)
        torch.cuda.current_stream().wait_stream(s)
        for _ in range(20):
            torch.mm(a, a)
        copies.append(K.clone())
        del K, V
        with torch.cuda.stream(s):
            [torch.full_like(want, 7.0) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(c, want) for c in copies)
