"""Attention over pages: how the ranges of a batch are given out (more than 64 sequences, one long among short ones), capped or biased pieces of a prompt over several ranges, and
scales and slopes at their ends, against 64 bits with bounds key by key."""
import pytest
import torch

from masked_bounds import attend_by_key, zero_would_fail
from masked_util import HALF_BF16, compare, paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as p
    p.lib()
    return p


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(vfa, g, lens, Hq, Hkv, d, page, n_q=1, cap=0.0, slopes=None, n_splits=None, number=False, holes=(), scale=None, sharp=1.5):
    rows, there, pool, table = paged(g, lens, Hkv, d, page, max(lens) + 37, holes=holes)
    B, gq = len(lens), Hq // Hkv
    q = (sharp * torch.randn((B, Hq, n_q, d), generator=g)).to(torch.bfloat16)
    kw = dict(score_cap=cap, slopes=None if slopes is None else torch.tensor(slopes, device="cuda"), n_splits=n_splits, **({} if scale is None else dict(softmax_scale=scale)))
    O, lse = vfa.kvp_decode_fwd(q.cuda(), tuple(p.cuda() for p in pool), table.cuda(), lens[0] if number else torch.tensor(lens, dtype=torch.int32, device="cuda"), **kw)
    O, lse = O.cpu(), lse.cpu()
    for b, n in enumerate(lens):
        pos, key = torch.arange(n - n_q, n)[:, None], torch.arange(n)[None]
        seen, away = (key <= pos) & there[b][None], (pos - key).abs().double()
        for h in range(Hq):
            k, v = (torch.where(there[b][:, None], x[h // gq], 0) for x in rows[b])
            want = attend_by_key(q[b, h], k, v, seen, away, cap, None if slopes is None else slopes[h], scale, weights=2.0 ** -15 if gq * n_q <= 16 else HALF_BF16)
            compare(O[b, h], lse[b, h], *want, (b, h, n))
            if n:
                assert zero_would_fail(*want[:3]), (b, h, n)


def lengths(g, B, most, longest):
    out = [int(x) for x in torch.randint(0, most, (B,), generator=g)]
    out[B // 3] = longest
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,n_splits", [(65, 2, 2, 2), (65, 4, 2, 5), (65, 2, 1, 30), (100, 2, 1, 8), (129, 3, 1, 12), (200, 1, 1, 3), (256, 2, 2, 4), (256, 20, 1, 2), (256, 2, 1, None),
                                               (257, 2, 1, 2), (100, 4, 4, None)])
def test_more_than_64_sequences(vfa, d, B, Hq, Hkv, n_splits):
    # (65 to 256: dealt to workgroups of one wave where there are at most eight ranges for each compute unit and the capacity has more than two tiles for each)
    g = gen(B + d)
    check(vfa, g, lengths(g, B, 150, 3000), Hq, Hkv, d, 16, n_splits=n_splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [63, 80, 150])
def test_one_long_sequence_among_short_ones(vfa, d, B):
    g = gen(B)
    check(vfa, g, lengths(g, B, 70, 9000), 4, 2, d, 64, cap=30.0, slopes=[0.01, 0.3, 0.0, -0.0005], holes={(B // 3, 5), (B // 3, 77), (0, 0)})


SLOPES = [0.5, 0.011, 1.7, 0.0, -0.003, 0.08, 0.2, 0.9]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", [(30.0, False), (0.0, True), (50.0, True)])
@pytest.mark.parametrize("n_q,n_splits", [(9, 3), (20, 4), (50, 2), (33, None), (5, 7)])
@pytest.mark.parametrize("lens,number", [([700, 40, 64, 333], False), ([500, 500], True), ([600], False)])
def test_scores_of_pieces_over_ranges(vfa, d, cap, bias, n_q, n_splits, lens, number):
    # (9 tokens of four heads: 36 rows, more than one group's)
    check(vfa, gen(int(cap) + n_q), lens, 8, 2, d, 16, n_q=n_q, cap=cap, slopes=SLOPES if bias else None, n_splits=n_splits, number=number, sharp=6.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
@pytest.mark.parametrize("n_q,n_splits", [(1, 1), (1, 4), (7, 2), (30, 2)])
def test_scales_and_slopes_at_the_ends(vfa, d, cap, n_q, n_splits):
    lens = [100, 200, 641]
    check(vfa, gen(3), lens, 8, 2, d, 16, n_q=n_q, cap=cap, slopes=SLOPES[:6] + [2.0 ** 18, -(2.0 ** 17)], scale=2.0 ** -64, n_splits=n_splits)
    check(vfa, gen(3), lens, 8, 2, d, 16, n_q=n_q, cap=cap, slopes=SLOPES, scale=2.0 ** 16, n_splits=n_splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
@pytest.mark.parametrize("n_q,n_splits", [(1, 1), (1, 3), (6, 2), (20, 2)])
def test_steep_biases_leave_one_key(vfa, d, cap, n_q, n_splits):
    # The newest key, at distance 0, has the weight 1, which is exact in any of its forms; the oldest one's may be rounded, and so is the output.
    g, n = gen(4), 500
    rows, _, pool, table = paged(g, [n, n], 2, d, 32, n)
    q = torch.randn((2, 4, n_q, d), generator=g).to(torch.bfloat16).cuda()
    cache, table, lens = tuple(p.cuda() for p in pool), table.cuda(), torch.tensor([n, n], dtype=torch.int32, device="cuda")
    v = torch.stack([rows[b][1] for b in range(2)]).repeat_interleave(2, 1)
    for sign, want in ((1, v[:, :, n - n_q:]), (-1, v[:, :, :1].expand(2, 4, n_q, d))):
        slopes = torch.full((4,), sign * 2.0 ** 18, device="cuda")
        O, _ = vfa.kvp_decode_fwd(q, cache, table, lens, score_cap=cap, slopes=slopes, softmax_scale=2.0 ** -64, n_splits=n_splits)
        if sign > 0:
            assert torch.equal(O.cpu(), want)
        else:
            assert ((O.cpu().double() - want.double()).abs() <= 1.01 * 2 * HALF_BF16 * want.double().abs()).all()
