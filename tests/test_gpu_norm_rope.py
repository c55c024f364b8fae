"""qk_norm_rope_fwd against 64 bits."""
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


def rnd(shape, seed, size=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * size).to(torch.bfloat16).cuda()


def table(n, rot, seed=0):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float().cuda()


def check(got, x, w, eps, cs, inter, first, norm):
    """One rounding to bf16; 2^-16 of the terms for the sum of squares (128 products) and a few more operations in 32 bits."""
    y, size = ref.norm_rope(x, w, eps, cs, inter, first, norm)
    off = (got.double().cpu() - y).abs() - 2.0 ** -8 * y.abs() - 2.0 ** -16 * size
    assert (off <= 0).all(), off.max().item()


@pytest.mark.parametrize("d,rot", [(64, 64), (64, 0), (64, 16), (64, 48), (128, 128), (128, 64), (128, 0), (128, 112)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_forms(vfa, d, rot, inter, norm):
    B, N, Hq, H = 2, 5, 6, 2
    x = rnd((B, N, Hq + 2 * H, d), rot, 3.0)
    w = (1 + 0.3 * rnd((2, d), 1)).to(torch.bfloat16) if norm else (None, None)
    cs = table(40, rot) if rot else None
    q, k, v = x[:, :, :Hq], x[:, :, Hq: Hq + H], x[:, :, Hq + H:]
    first = [3, 33]
    Q, K, V = vfa.qk_norm_rope_fwd(q, k, v, norm=norm, q_weight=w[0], k_weight=w[1], eps=1e-5, cos_sin=cs, interleaved=inter,
                                   first_pos=torch.tensor(first, dtype=torch.int32, device="cuda"))
    check(Q, q, w[0], 1e-5, cs, inter, first, norm)
    check(K, k, w[1], 1e-5, cs, inter, first, norm)
    assert torch.equal(V, v.transpose(1, 2))


@pytest.mark.parametrize("B,N,Hq,H", [(1, 1, 1, 1), (1, 1, 32, 8), (16, 1, 8, 1), (3, 33, 5, 5), (1, 100, 12, 3), (2, 65, 64, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_shapes(vfa, B, N, Hq, H, d):
    q, k = rnd((B, N, Hq, d), 1), rnd((B, N, H, d), 2, 1e-3)
    w = (1 + 0.3 * rnd((d,), 1)).to(torch.bfloat16)
    cs = table(N + 7, d)
    Q, K, V = vfa.qk_norm_rope_fwd(q, k, q_weight=w, cos_sin=cs, first_pos=4)
    assert V is None
    check(Q, q, w, 1e-6, cs, False, [4] * B, True)
    check(K, k, None, 1e-6, cs, False, [4] * B, True)


def test_positions_are_clamped(vfa):
    q = rnd((3, 4, 2, 64), 3)
    cs = table(6, 64)
    first = [-2, 4, 1000000]
    Q, K, _ = vfa.qk_norm_rope_fwd(q, q, norm=False, cos_sin=cs, first_pos=torch.tensor(first, dtype=torch.int32, device="cuda"))
    check(Q, q, None, 0.0, cs, False, first, False)
    assert torch.equal(Q, K)
    Q, _, _ = vfa.qk_norm_rope_fwd(q, q, norm=False, cos_sin=cs, first_pos=-1)
    check(Q, q, None, 0.0, cs, False, [-1] * 3, False)
    top = 2 ** 31 - 1
    Q, _, _ = vfa.qk_norm_rope_fwd(q, q, norm=False, cos_sin=cs, first_pos=top)
    check(Q, q, None, 0.0, cs, False, [top] * 3, False)


def test_strides_and_outputs(vfa):
    """A head axis of stride zero, a transposed projection, outputs that the caller gives."""
    B, N, H, d = 2, 9, 4, 128
    x = rnd((N, B, H, d), 4).transpose(0, 1)
    one = rnd((B, N, 1, d), 5).expand(B, N, H, d)
    out = [torch.full((B, H, N, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    got = vfa.qk_norm_rope_fwd(x, one, x, out=out)
    check(out[0], x, None, 1e-6, None, False, None, True)
    check(out[1], one, None, 1e-6, None, False, None, True)
    assert torch.equal(out[2], x.transpose(1, 2)) and all(a is b for a, b in zip(got, out))


def test_rows_of_zeros_large_and_small(vfa):
    x = rnd((1, 4, 2, 64), 6)
    x[:, 1] = 0
    x[:, 2] *= 2.0 ** 40
    x[:, 3] *= 2.0 ** -40
    Q, _, _ = vfa.qk_norm_rope_fwd(x, x, eps=1e-6)
    check(Q, x, None, 1e-6, None, False, None, True)
    Q, _, _ = vfa.qk_norm_rope_fwd(x[:, 2:], x[:, 2:], eps=0.0)
    check(Q, x[:, 2:], None, 0.0, None, False, None, True)
    x[0, 0, 0, 3], x[0, 1, 0, 0] = float("nan"), float("inf")
    Q, _, _ = vfa.qk_norm_rope_fwd(x, x, eps=1e-6)
    assert Q[0, 0, 0].isnan().all() and Q[0, 0, 1, 0].isnan() and not Q[0, 1].isnan().any() and not Q[0, 0, 2:].isnan().any()


def test_empty(vfa):
    q = torch.empty((0, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    Q, K, _ = vfa.qk_norm_rope_fwd(q, q)
    assert Q.shape == (0, 2, 3, 64)
    q = torch.empty((3, 0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert vfa.qk_norm_rope_fwd(q, q)[1].shape == (3, 2, 0, 64)


@pytest.mark.parametrize("d,rot", [(64, 16), (64, 48), (128, 16), (128, 64), (128, 112)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_unrotated_features_stand_alone(vfa, d, rot, inter, norm):
    """An infinity or NaN in each unrotated feature of a token in turn: without the norm no other feature changes, with it an infinity leaves
    zeros beside it."""
    kinds = [float("inf"), float("-inf"), float("nan")]
    N = 3 * (d - rot)
    clean = rnd((1, N, 3, d), rot, 3.0)
    x = clean.clone()
    at = [rot + n // 3 for n in range(N)]
    for n in range(N):
        x[0, n, 1, at[n]] = kinds[n % 3]
    cs = table(N + 2, rot)
    Q, K, _ = vfa.qk_norm_rope_fwd(x, x, norm=norm, eps=1e-5, cos_sin=cs, interleaved=inter, first_pos=2)
    assert torch.equal(Q.nan_to_num(7.0), K.nan_to_num(7.0))
    y, size = ref.norm_rope(x, None, 1e-5, cs, inter, [2], norm)
    got = Q.double().cpu()
    assert torch.equal(got.isnan(), y.isnan()) and torch.equal(got.isinf(), y.isinf())
    fin = y.isfinite()
    off = (got - y).abs() - 2.0 ** -8 * y.abs() - 2.0 ** -16 * size
    assert (off[fin] <= 0).all(), off[fin].max().item()
    if not norm:
        same = vfa.qk_norm_rope_fwd(clean, clean, norm=False, cos_sin=cs, interleaved=inter, first_pos=2)[0]
        for n in range(N):
            same[0, 1, n, at[n]] = x[0, n, 1, at[n]]
        assert torch.equal(Q.nan_to_num(7.0), same.nan_to_num(7.0))
