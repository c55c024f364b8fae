"""Masked, capped or biased prompts of so many rows that a workgroup takes 128 of them (fewer give it 64, which the other tests of masked attention run): sizes, masks,
special values, ends of scales, and the order of the items, against 64 bits."""
import math
import random

import pytest
import torch

from masked_bounds import attend_by_key, zero_would_fail
from masked_util import compare
from test_gpu_masked_attn import SCORES, documents, ints, prompt, ranges_of

pytestmark = pytest.mark.gpu

SLOPES = [0.5, 0.011, 1.7, -0.003, 0.0, 0.06]


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as p
    p.lib()
    return p


def places(d):
    """Workgroups of 128 rows that the GPU holds at once; from as many on they are taken (tests/test_masked_launches.py)."""
    return (3 if d == 64 else 2) * torch.cuda.get_device_properties(0).multi_processor_count


def heads(N, d, g=2, unit=1, B=2):
    """(Hq, Hkv) so that B of them are just enough; Hkv a multiple of `unit`."""
    Hkv = -(-places(d) // (B * g * -(-N // 128)))
    Hkv = -(-Hkv // unit) * unit
    return g * Hkv, Hkv


def slopes_of(Hq, slopes=SLOPES):
    return [slopes[h % len(slopes)] for h in range(Hq)]


def sample(rng, n, some):
    return sorted({0, n - 1, *(rng.randrange(n) for _ in range(some))})


def run(vfa, Q, K, V, causal=None, ranges=None, cap=0.0, slopes=None, scale=None):
    B, Hq, N, d = Q.shape
    assert B * Hq * -(-N // 128) >= places(d), "too few rows for workgroups of 128"
    kw = {} if scale is None else dict(softmax_scale=scale)
    s = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
    return vfa.masked_attn_fwd(Q.cuda(), K.cuda(), V.cuda(), causal=causal, ranges=None if ranges is None else ranges.cuda(), score_cap=cap, slopes=s, **kw)


def seen_by(rows, N, b, causal, ranges):
    key = torch.arange(N, device=rows.device)[None]
    seen = torch.ones((len(rows), N), dtype=torch.bool, device=rows.device)
    if ranges is not None:
        r = ranges[b].to(rows.device)[rows]
        seen = (key >= r[:, :1]) & (key < r[:, 1:])
    if causal or (causal is None and ranges is None):
        seen = seen & (key <= rows[:, None])
    return seen


def check(vfa, Q, K, V, causal=None, ranges=None, cap=0.0, slopes=None, scale=None, what="", finite=True):
    O, lse = run(vfa, Q, K, V, causal, ranges, cap, slopes, scale)
    B, Hq, N, d = Q.shape
    g = Hq // K.shape[1]
    rng = random.Random(N + d)
    for b in range(B):
        rows = torch.tensor(sample(rng, N, 60))
        seen = seen_by(rows, N, b, causal, ranges)
        away = (rows[:, None] - torch.arange(N)[None]).abs().double()
        for h in sample(rng, Hq, 4):
            want = attend_by_key(Q[b, h, rows], K[b, h // g], V[b, h // g], seen, away, cap, None if slopes is None else slopes[h], scale)
            compare(O[b, h, rows], lse[b, h, rows], *want, (what, b, h))
            assert not finite or zero_would_fail(want[0], want[1], want[2]), (what, b, h)
    return O, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 31, 64, 127, 128, 129, 333, 640, 1100])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("causal", [True, False])
def test_whole(vfa, d, N, cap, bias, causal):
    Hq, Hkv = heads(N, d)
    check(vfa, *prompt(N, 2, Hq, Hkv, N, d, 6.0 if cap else 1.5), causal=causal, cap=cap, slopes=slopes_of(Hq) if bias else None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,n_docs", [(128, 2), (129, 10), (500, 7), (777, 3), (300, 300), (1500, 4)])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("causal,prefix", [(True, False), (True, True), (False, False)])
def test_documents(vfa, d, N, n_docs, cap, bias, causal, prefix):
    rng = random.Random(N + n_docs)
    offsets = [documents(rng, N, n_docs, pad) for pad in (0, N // 4)]
    pre = [[rng.randint(0, 400) for _ in range(n_docs)] for _ in offsets] if prefix else None
    ranges = vfa.row_ranges(ints(offsets), N, prefix_lens=ints(pre) if prefix else None, causal=causal).cpu()
    assert torch.equal(ranges, ranges_of(offsets, pre, N, causal))
    Hq, Hkv = heads(N, d, unit=4)
    check(vfa, *prompt(N, 2, Hq, Hkv, N, d, 6.0 if cap else 1.5), ranges=ranges, cap=cap, slopes=slopes_of(Hq) if bias else None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", SCORES)
def test_any_ranges(vfa, d, cap, bias):
    """Windows, runs of keys behind or before the row, empty rows, ends outside of the sequence, with and without a causal mask on top."""
    N, rng = 700, random.Random(4)
    any_ = [[(a, a + rng.choice([0, 1, 3, 64, 65, 300, -4])) for a in [rng.randint(-20, N + 20) for _ in range(N)]] for _ in range(2)]
    window = [[(max(0, i - 270), i + 1) for i in range(N)], [(0, 0) if 100 <= i < 400 else (i - 5, i + 190) for i in range(N)]]
    ends = [[(-2 ** 31, 2 ** 31 - 1)] * N, [(2 ** 31 - 1, -2 ** 31)] * (N // 2) + [(N - 1, N)] * (N // 2)]
    tail = [[(N - 129, N)] * N, [(500, 600)] * N]  # (all keys behind most of the rows)
    Hq, Hkv = heads(N, d, g=1)
    Q, K, V = prompt(1, 2, Hq, Hkv, N, d)
    for what, r in (("any", any_), ("window", window), ("ends", ends), ("tail", tail)):
        for causal in (True, None):
            check(vfa, Q, K, V, ranges=torch.tensor(r, dtype=torch.int32), causal=causal, cap=cap, slopes=slopes_of(Hq) if bias else None, what=what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("x", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("cap,bias", SCORES)
def test_special_values_stay_in_their_document(vfa, d, x, cap, bias):
    """NaN and infinities of a document, or of padding, reach no other one: those have the bits that they have without."""
    N, o = 900, [0, 100, 130, 131, 533, 650]
    Hq, Hkv = heads(N, d)
    Q, K, V = (t.cuda() for t in prompt(d, 2, Hq, Hkv, N, d))
    ranges = vfa.row_ranges(ints([o, [0, 5, 200, 333, 600, N]]), N)
    kw = dict(ranges=ranges, cap=cap, slopes=slopes_of(Hq) if bias else None)
    clean, clean_l = run(vfa, Q, K, V, **kw)
    for lo, hi in ((100, 130), (130, 131), (131, 533), (650, N), (0, 100)):
        k, v, q = K.clone(), V.clone(), Q.clone()
        v[0, :, lo:hi, ::3] = x
        k[0, :, lo:hi] = x
        q[0, :, lo:hi] = x
        O, lse = run(vfa, q, k, v, **kw)
        keep = torch.ones((2, N), dtype=torch.bool, device="cuda")
        keep[0, lo:hi] = False
        for a, b in ((O, clean), (lse, clean_l)):
            assert torch.equal(a.transpose(1, 2)[keep], b.transpose(1, 2)[keep]), (lo, hi)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_special_values_behind_a_row(vfa, d, cap):
    """Values that are not finite reach the rows that see their key, and no others: causal, prefixes, all."""
    N = 900
    Hq, Hkv = heads(N, d)
    Q, K, V = prompt(d, 2, Hq, Hkv, N, d)
    for t, f, x in ((40, 3, math.inf), (41, 3, -math.inf), (70, 5, math.nan), (150, 7, math.inf), (290, 9, -math.inf), (290, 10, math.nan), (128, 11, math.inf),
                    (600, 12, math.nan), (895, 13, math.inf)):
        V[:, :, t, f::32] = x
    check(vfa, Q, K, V, cap=cap, finite=False)
    offsets = [[0, 45, 400, N], [0, 300, 301, 880]]
    check(vfa, Q, K, V, ranges=vfa.row_ranges(ints(offsets), N, prefix_lens=ints([[42, 200, 95], [300, 0, 250]])).cpu(), cap=cap, finite=False)
    check(vfa, Q, K, V, ranges=vfa.row_ranges(ints(offsets), N, causal=False).cpu(), cap=cap, finite=False)
    # NaN among the keys behind every row that is compared
    K[:, :, 700:] = math.nan
    O, lse = run(vfa, Q, K, V, cap=cap)
    assert O[:, :, :700, 20].isfinite().all() and lse[:, :, :700].isfinite().all() and lse[:, :, 700:].isnan().all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("N", [1, 200, 700])
def test_rows_that_see_one_key_get_its_value(vfa, d, cap, bias, N):
    # its weight is a power of two and the sum that weight within 2^-16, far below half a step of bf16
    Hq, Hkv = heads(N, d)
    Q, K, V = (x.cuda() for x in prompt(N, 2, Hq, Hkv, N, d))
    key = torch.randint(0, N, (2, N), generator=torch.Generator().manual_seed(N)).int()
    O, _ = run(vfa, Q, K, V, causal=False, ranges=torch.stack((key, key + 1), -1), cap=cap, slopes=slopes_of(Hq) if bias else None)
    at = key.cuda().long()[:, None, :, None].expand(2, Hq, N, d)
    assert torch.equal(O, V.repeat_interleave(2, 1).gather(2, at))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
def test_scales_and_slopes_at_the_ends(vfa, d, cap):
    for N in (40, 500):
        Hq, Hkv = heads(N, d)
        Q, K, V = prompt(7, 2, Hq, Hkv, N, d)
        for what, causal, scale, slopes in (("steep", None, 2.0 ** -64, [0.3, 2.0 ** 18]), ("steep both ways", False, 2.0 ** -64, [-(2.0 ** 18), 2.0 ** 12]),
                                            ("large scale", None, 2.0 ** 16, [0.3, 0.0])):
            check(vfa, Q, K, V, causal=causal, scale=scale, cap=cap, slopes=slopes_of(Hq, slopes), what=what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
def test_steep_biases_leave_one_key(vfa, d, cap):
    # A steep bias leaves the row itself, whose distance is 0 and whose weight so is a power of two.  The other way round it leaves the farthest key: its weight is rounded
    # to bf16 and so is the output, the sum that divides is the weight itself.
    N = 500
    Hq, Hkv = heads(N, d, g=1)
    Q, K, V = (x.cuda() for x in prompt(8, 2, Hq, Hkv, N, d))
    for causal in (True, False):
        O, _ = run(vfa, Q, K, V, causal=causal, scale=2.0 ** -64, cap=cap, slopes=[2.0 ** 18] * Hq)
        assert torch.equal(O, V), causal
        O, _ = run(vfa, Q, K, V, causal=causal, scale=2.0 ** -64, cap=cap, slopes=[-(2.0 ** 18)] * Hq)
        far = torch.arange(N, device="cuda")
        want = V[:, :, torch.where(far > N - 1 - far, 0, 0 if causal else N - 1)].double()
        assert ((O.double() - want).abs() <= 1.01 * 2 * 2.0 ** -8 * want.abs()).all(), causal


@pytest.mark.parametrize("cap", [20.0, 43.0, 50.0, 100.0, 1000.0])
def test_capped_scores_at_both_ends(vfa, cap):
    """All scores at -cap, all at +cap, and some of each: a row's max may be anywhere."""
    N, d = 400, 128
    Hq, Hkv = heads(N, d, g=1)
    Q, K, V = prompt(3, 2, Hq, Hkv, N, d)
    Q, K = Q.abs() * 8, K.abs() * 8
    K[:, :, :150] *= -1
    for what, k, slopes in (("the last", K, None), ("the first", -K, None), ("none", -K.abs(), None), ("all, biased", K.abs(), [0.0, 1.0])):
        check(vfa, Q, k, V, cap=cap, slopes=slopes and slopes_of(Hq, slopes), what=what)


@pytest.mark.parametrize("B,Hq,Hkv,N,d,parts", [(5, 64, 8, 1000, 128, [3, 2]), (7, 64, 8, 800, 128, [3, 3, 1]), (5, 128, 8, 600, 64, [3, 2]), (1, 60, 5, 1700, 128, []), (3, 63, 9, 1500, 64, [])])
def test_every_row_of_every_head(vfa, B, Hq, Hkv, N, d, parts):
    """Where the GPU is filled more than twice over, an XCD's KV heads are taken some at a time, the last time fewer; each item is somebody's, once."""
    items, at_once = B * Hq * -(-N // 128), places(d)
    if parts and torch.cuda.get_device_properties(0).multi_processor_count == 256:
        n = items // (2 * at_once)
        assert len(parts) == n and parts[0] == -(-B * Hkv // 8 // n) and sum(parts) == B * Hkv // 8
    Q, K, V = (x.cuda() for x in prompt(N, B, Hq, Hkv, N, d))
    rng = random.Random(N)
    ranges = vfa.row_ranges(ints([documents(rng, N, 3, N // 9) for _ in range(B)]), N) if B % 2 else None
    O = torch.full_like(Q, math.nan)
    assert items >= at_once
    _, lse = vfa.masked_attn_fwd(Q, K, V, ranges=ranges, out=O)
    rows, g = torch.arange(N, device="cuda"), Hq // Hkv
    for b in range(B):
        seen = seen_by(rows, N, b, None, ranges)
        for h in range(Hkv):
            mine = slice(h * g, h * g + g)
            want = attend_by_key(Q[b, mine].reshape(-1, d), K[b, h], V[b, h], seen.repeat(g, 1), None, 0.0, None)
            compare(O[b, mine].reshape(-1, d), lse[b, mine].reshape(-1), *(t.cpu() for t in want), (b, h))


@pytest.mark.parametrize("d", [64, 128])
def test_longest(vfa, d):
    """The longest prompt that is taken: a head's keys end one row short of 2^31 bytes.  Windows, so that it takes no time; rows at either end and between."""
    N = 0x7FFFFFFF // (2 * d)
    g = torch.Generator("cuda").manual_seed(d)
    Q, K, V = (torch.randn((1, 1, N, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    i = torch.arange(N, device="cuda", dtype=torch.int32)
    ranges = torch.stack((i - 150, i + 60), -1)[None].contiguous()
    assert -(-N // 128) >= places(d)
    O, lse = vfa.masked_attn_fwd(Q, K, V, ranges=ranges, slopes=torch.tensor([0.02], device="cuda"))
    for r in (0, 127, N // 3, N // 2 + 1, N - 128, N - 40, N - 1):
        lo, hi = max(0, r - 150), min(N, r + 60)
        key = torch.arange(lo, hi)
        seen = torch.ones((1, hi - lo), dtype=torch.bool)
        want = attend_by_key(Q[0, 0, r: r + 1].cpu(), K[0, 0, lo:hi].cpu(), V[0, 0, lo:hi].cpu(), seen, (r - key).abs().double()[None], 0.0, 0.02)
        compare(O[0, 0, r: r + 1], lse[0, 0, r: r + 1], *want, r)
    with pytest.raises(vfa.VfaError):
        vfa.masked_attn_fwd(*(torch.empty((1, 1, N + 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)))


def test_replayed(vfa):
    """Captured once and replayed with new inputs and masks, an eager call of the same kind between the replays."""
    N, d = 600, 128
    Hq, Hkv = heads(N, d)
    g = torch.Generator().manual_seed(0)
    Q, K, V = (torch.zeros((2, h, N, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    ranges, O, L = torch.zeros((2, N, 2), dtype=torch.int32, device="cuda"), torch.empty_like(Q), torch.empty((2, Hq, N), device="cuda")
    slopes, offsets = torch.tensor(slopes_of(Hq), device="cuda"), ints([[0, 5, N]] * 2)
    assert 2 * Hq * -(-N // 128) >= places(d)

    def work():
        vfa.row_ranges(offsets, N, out=ranges)
        vfa.masked_attn_fwd(Q, K, V, ranges=ranges, score_cap=30.0, slopes=slopes, out=O, lse=L)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        for t in (Q, K, V):
            t.copy_(torch.randn(t.shape, generator=g))
        offsets.copy_(torch.tensor([[0, 60 + turn, N - turn], [turn, 128, 530]]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen = O.clone(), L.clone()
        for t in (O, L):
            t.fill_(math.nan)
        work()
        torch.cuda.synchronize()
        assert torch.equal(seen[0], O) and torch.equal(seen[1], L), turn
