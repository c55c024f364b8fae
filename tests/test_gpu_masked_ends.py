"""Masked attention of few rows (workgroups of 64) at the ends of its scales and slopes, with bounds key by key: an error that a far key of weight zero may have allows nothing."""
import random

import pytest
import torch

from masked_bounds import attend_by_key, zero_would_fail
from masked_util import HALF_BF16, compare
from test_gpu_masked_attn import SCORES, documents, prompt, ranges_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as p
    p.lib()
    return p


def check(vfa, Q, K, V, causal=True, ranges=None, cap=0.0, slopes=None, scale=None, what=""):
    B, Hq, N, d = Q.shape
    s = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
    O, lse = vfa.masked_attn_fwd(Q.cuda(), K.cuda(), V.cuda(), causal=causal, ranges=None if ranges is None else ranges.cuda(), score_cap=cap, slopes=s,
                                 **({} if scale is None else dict(softmax_scale=scale)))
    i = torch.arange(N)
    away = (i[:, None] - i[None]).abs().double()
    for b in range(B):
        seen = i[None] <= (i[:, None] if causal else N)
        if ranges is not None:
            seen = seen & (i[None] >= ranges[b, :, :1]) & (i[None] < ranges[b, :, 1:])
        for h in range(Hq):
            want = attend_by_key(Q[b, h], K[b, h * K.shape[1] // Hq], V[b, h * K.shape[1] // Hq], seen, away, cap, None if slopes is None else slopes[h], scale)
            compare(O[b, h], lse[b, h], *want, (what, b, h))
            assert zero_would_fail(*want[:3]), (what, b, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
@pytest.mark.parametrize("N", [40, 97, 500])
def test_scales_and_slopes_at_the_ends(vfa, d, cap, N):
    for what, causal, scale, slopes in (("steep", True, 2.0 ** -64, [0.3, 2.0 ** 18]), ("steep both ways", False, 2.0 ** -64, [-(2.0 ** 18), 2.0 ** 12]),
                                        ("large scale", True, 2.0 ** 16, [0.3, 0.0])):
        check(vfa, *prompt(7, 1, 2, 1, N, d), causal=causal, scale=scale, cap=cap, slopes=slopes, what=what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
def test_steep_biases_leave_one_key(vfa, d, cap):
    # as on workgroups of 128 rows: the row's own value to the bit, the farthest key's within two roundings
    N = 500
    Q, K, V = (x.cuda() for x in prompt(8, 2, 2, 2, N, d))
    for causal in (True, False):
        O, _ = vfa.masked_attn_fwd(Q, K, V, causal=causal, softmax_scale=2.0 ** -64, score_cap=cap, slopes=torch.full((2,), 2.0 ** 18, device="cuda"))
        assert torch.equal(O, V), causal
        O, _ = vfa.masked_attn_fwd(Q, K, V, causal=causal, softmax_scale=2.0 ** -64, score_cap=cap, slopes=torch.full((2,), -(2.0 ** 18), device="cuda"))
        far = torch.arange(N, device="cuda")
        want = V[:, :, torch.where(far > N - 1 - far, 0, 0 if causal else N - 1)].double()
        assert ((O.double() - want).abs() <= 1.01 * 2 * HALF_BF16 * want.abs()).all(), causal


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("N", [33, 300])
def test_documents(vfa, d, cap, bias, N):
    rng = random.Random(N)
    offsets = [documents(rng, N, 4, pad) for pad in (0, N // 4)]
    check(vfa, *prompt(N, 2, 4, 2, N, d, 6.0 if cap else 1.5), causal=False, ranges=ranges_of(offsets, None, N, True), cap=cap, slopes=[3.0, -2.7, 40.0, 0.01] if bias else None)
