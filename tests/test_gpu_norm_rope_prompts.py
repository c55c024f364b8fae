"""qk_norm_rope_fwd on prompts: four heads of a thread (where that still gives two workgroups for each compute unit), and loads and stores past the caches
(from 2^26 elements on, d = 128).  Tokens drawn from all of them and both ends against 64 bits, values and what was not rotated bit for bit."""
import pytest
import torch

import kv8_util as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2604_12798_amd as pkg
    pkg.lib()
    return pkg


def table(n, rot):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float().cuda()


def check(vfa, B, N, Hq, H, d, rot, inter, norm, values=True, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, N, Hq + 2 * H, d), generator=g, device="cuda", dtype=torch.bfloat16) * 3
    w = (1 + 0.3 * torch.randn((2, d), generator=g, device="cuda")).to(torch.bfloat16) if norm else (None, None)
    q, k, v = x[:, :, :Hq], x[:, :, Hq: Hq + H], x[:, :, Hq + H:]
    cs = table(N + 50, rot) if rot else None
    first = [7 * b for b in range(B)]
    out = [torch.full((B, h, N, d), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H)]
    got = vfa.qk_norm_rope_fwd(q, k, v if values else None, norm=norm, q_weight=w[0], k_weight=w[1], eps=1e-5, cos_sin=cs, interleaved=inter,
                               first_pos=torch.tensor(first, dtype=torch.int32, device="cuda"), out=out if values else None)
    assert not any(t.isnan().any() for t in got if t is not None)  # (every row was written)
    if values:
        assert torch.equal(got[2], v.transpose(1, 2))
    else:
        assert got[2] is None
    tokens = sorted({0, 1, 63, 64, N - 2, N - 1, *torch.randint(0, N, (12,), generator=torch.Generator().manual_seed(seed)).tolist()})
    for n in tokens:
        for t, src, weight in ((got[0], q, w[0]), (got[1], k, w[1])):
            y, size = ref.norm_rope(src[:, n: n + 1], weight, 1e-5, cs, inter, [f + n for f in first], norm)
            # (one rounding to bf16; 2^-16 of the terms for the sum of squares and a few more operations in 32 bits)
            off = (t[:, :, n: n + 1].double().cpu() - y).abs() - 2.0 ** -8 * y.abs() - 2.0 ** -16 * size
            assert (off <= 0).all(), (n, off.max().item())
    if not norm:
        for t, src in ((got[0], q), (got[1], k)):
            assert torch.equal(t[..., rot:], src.transpose(1, 2)[..., rot:])


# 5 + 3 + 3 heads: a thread's four begin with queries and end with keys, begin with keys and end with values, and the last has three; 6 + 1 + 1: queries, keys and
# values in one thread's; 5 + 3 without values: two whole ones.  Tokens are no multiple of a workgroup's 32 (d = 128) or 64.
@pytest.mark.parametrize("B,N,Hq,H,values", [(2, 6001, 5, 3, True), (1, 17003, 6, 1, True), (3, 9001, 5, 3, False)])
@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (64, 32, True), (64, 16, False), (64, 0, False), (128, 128, False), (128, 128, True), (128, 48, False),
                                         (128, 64, True), (128, 0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_four_heads_of_a_thread(vfa, B, N, Hq, H, values, d, rot, inter, norm):
    check(vfa, B, N, Hq, H, d, rot, inter, norm, values, seed=d + rot)


# the smallest that go past the caches, and the same with one token less; a half that is rotated in pairs (i, i + 32) does not
@pytest.mark.parametrize("N", [47662, 47663])
@pytest.mark.parametrize("rot,inter", [(128, False), (128, True), (64, True), (64, False), (0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_past_the_caches(vfa, N, rot, inter, norm):
    check(vfa, 1, N, 5, 3, 128, rot, inter, norm, seed=rot + N)
