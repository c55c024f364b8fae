"""Prompts with ranges of their own for each row, capped or biased scores, and the ranges of documents and prefixes, against 64 bits."""
import math
import random

import pytest
import torch

from masked_util import attend, compare, paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as p
    p.lib()
    return p


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- ranges ----------------------------------------------------------------------------------------------------------------------

def ranges_of(offsets, prefix, N, causal):
    out = []
    for b, o in enumerate(offsets):
        o = [min(max(x, 0), N) for x in o]
        rows = [(0, 0)] * N
        for k in range(len(o) - 1):
            for i in range(o[k], o[k + 1]):
                rows[i] = (o[k], max(i + 1, min(o[k] + (prefix[b][k] if prefix else 0), o[k + 1])) if causal else o[k + 1])
        out.append(rows)
    return torch.tensor(out, dtype=torch.int32).reshape(len(offsets), N, 2)


def documents(rng, N, n, pad=0):
    end = N - pad
    return [0] + sorted(rng.randint(0, end) for _ in range(n - 1)) + [end]


@pytest.mark.parametrize("N", [1, 2, 255, 256, 257, 1000, 5000])
@pytest.mark.parametrize("n_docs", [1, 2, 3, 30, 1023, 1024, 2500])
@pytest.mark.parametrize("causal", [True, False])
def test_row_ranges(vfa, N, n_docs, causal):
    rng = random.Random(N * n_docs)
    offsets = [documents(rng, N, n_docs, pad) for pad in (0, N // 3)]
    offsets[1][0] = offsets[1][1] // 2   # (rows in front of the first document)
    prefix = [[rng.choice([0, 1, 5, 300, 2 ** 31 - 1, -7]) for _ in range(n_docs)] for _ in offsets]
    for pre in (None, prefix):
        got = vfa.row_ranges(ints(offsets), N, prefix_lens=None if pre is None else ints(pre), causal=causal)
        assert torch.equal(got.cpu(), ranges_of(offsets, pre, N, causal)), (N, n_docs, pre is None)


def test_row_ranges_at_the_ends(vfa):
    for offsets in ([[-5, 3, 2 ** 31 - 1]], [[10, 20, 30]], [[4, 4, 4]], [[0, 0, 0]], [[7]], [[-2 ** 31, 12, 12, 2 ** 31 - 1]]):
        assert torch.equal(vfa.row_ranges(ints(offsets), 12).cpu(), ranges_of(offsets, None, 12, True)), offsets
    assert vfa.row_ranges(ints([[0, 3]]), 0).shape == (1, 0, 2)
    assert vfa.row_ranges(ints([[0, 3]])[:0], 5).shape == (0, 5, 2)
    out = torch.full((1, 5, 2), 9, dtype=torch.int32, device="cuda")
    assert vfa.row_ranges(ints([[0, 3]]), 5, out=out) is out and out[0, 4].tolist() == [0, 0]


# ---- prompts ---------------------------------------------------------------------------------------------------------------------

def prompt(seed, B, Hq, Hkv, N, d, sharp=1.5):
    g = torch.Generator().manual_seed(seed)
    mk = lambda h: torch.randn((B, h, N, d), generator=g)
    return (sharp * mk(Hq)).to(torch.bfloat16), mk(Hkv).to(torch.bfloat16), mk(Hkv).to(torch.bfloat16)


def check(vfa, Q, K, V, causal=None, ranges=None, cap=0.0, slopes=None, scale=None, rows=None):
    B, Hq, N, d = Q.shape
    s = None if slopes is None else torch.tensor(slopes, dtype=torch.float32)
    kw = dict(score_cap=cap, slopes=None if s is None else s.cuda(), ranges=None if ranges is None else ranges.cuda(), **({} if scale is None else dict(softmax_scale=scale)))
    O, lse = vfa.masked_attn_fwd(Q.cuda(), K.cuda(), V.cuda(), causal=causal, **kw)
    r = torch.arange(N) if rows is None else rows
    key = torch.arange(N)[None]
    away = (r[:, None] - key).abs().double()
    for b in range(B):
        seen = torch.ones((len(r), N), dtype=torch.bool)
        if ranges is not None:
            seen = (key >= ranges[b, r, :1]) & (key < ranges[b, r, 1:])
        if causal or (causal is None and ranges is None):
            seen = seen & (key <= r[:, None])
        for h in range(Hq):
            want = attend(Q[b, h, r], K[b, h * K.shape[1] // Hq], V[b, h * K.shape[1] // Hq], seen, away, cap, None if s is None else float(s[h]), scale)
            compare(O[b, h, r], lse[b, h, r], *want, (b, h))
    return O, lse


SIZES = [1, 2, 31, 63, 64, 65, 127, 128, 129, 200, 333, 640]
SCORES = [(0.0, False), (30.0, False), (0.0, True), (50.0, True)]
SLOPES = [0.5, 0.011, 1.7, -0.003]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", SIZES)
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("causal", [True, False])
def test_whole(vfa, d, N, cap, bias, causal):
    check(vfa, *prompt(N, 2, 4, 2, N, d, 6.0 if cap else 1.5), causal=causal, cap=cap, slopes=SLOPES if bias else None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,n_docs", [(64, 3), (128, 2), (129, 10), (500, 7), (777, 40), (300, 300)])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("causal,prefix", [(True, False), (True, True), (False, False)])
def test_documents(vfa, d, N, n_docs, cap, bias, causal, prefix):
    rng = random.Random(N + n_docs)
    offsets = [documents(rng, N, n_docs, pad) for pad in (0, N // 4)]
    pre = [[rng.randint(0, 100) for _ in range(n_docs)] for _ in offsets] if prefix else None
    ranges = vfa.row_ranges(ints(offsets), N, prefix_lens=ints(pre) if prefix else None, causal=causal)
    assert torch.equal(ranges.cpu(), ranges_of(offsets, pre, N, causal))
    check(vfa, *prompt(N, 2, 4, 2, N, d, 6.0 if cap else 1.5), ranges=ranges.cpu(), cap=cap, slopes=SLOPES if bias else None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bias", [False, True])
def test_any_ranges(vfa, d, bias):
    """Windows, runs of keys behind or before the row, empty rows, ends outside of the sequence, with and without a causal mask on top."""
    N, rng = 400, random.Random(4)
    any_ = [[(a, a + rng.choice([0, 1, 3, 64, 65, 200, -4])) for a in [rng.randint(-20, N + 20) for _ in range(N)]] for _ in range(2)]
    window = [[(max(0, i - 70), i + 1) for i in range(N)], [(0, 0) if 100 <= i < 300 else (i - 5, i + 9) for i in range(N)]]
    ends = [[(-2 ** 31, 2 ** 31 - 1)] * N, [(2 ** 31 - 1, -2 ** 31)] * (N // 2) + [(N - 1, N)] * (N // 2)]
    for r in (any_, window, ends):
        for causal in (True, False, None):
            check(vfa, *prompt(1, 2, 4, 4, N, d), ranges=torch.tensor(r, dtype=torch.int32), causal=causal, slopes=SLOPES if bias else None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_steep_biases_on_short_documents(vfa, d, cap):
    # the bias of a key's place in its block of 32 is far above the scores there
    rng = random.Random(d)
    for N in (5, 33, 44, 97, 600):
        offsets = [documents(rng, N, 4) for _ in range(2)]
        check(vfa, *prompt(N, 2, 4, 2, N, d, 0.1), ranges=ranges_of(offsets, None, N, True), cap=cap, slopes=[3.0, -2.7, 40.0, 0.9])


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (6, 3), (16, 8), (9, 9)])
def test_heads(vfa, Hq, Hkv):
    check(vfa, *prompt(Hq, 3, Hq, Hkv, 150, 128), slopes=[0.01 * h for h in range(Hq)])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("N", [1, 40, 333])
def test_rows_that_see_one_key_get_its_value(vfa, d, cap, bias, N):
    # its weight is a power of two and the sum that weight within 2^-16, far below half a step of bf16
    Q, K, V = (x.cuda() for x in prompt(N, 2, 4, 2, N, d))
    key = torch.randint(0, N, (2, N), generator=torch.Generator().manual_seed(N)).int()
    slopes = torch.tensor(SLOPES, device="cuda") if bias else None
    O, _ = vfa.masked_attn_fwd(Q, K, V, causal=False, ranges=torch.stack((key, key + 1), -1).cuda(), score_cap=cap, slopes=slopes)
    at = key.cuda().long()[:, None, :, None].expand(2, 4, N, d)
    assert torch.equal(O, V.repeat_interleave(2, 1).gather(2, at))


def test_scale(vfa):
    check(vfa, *prompt(7, 1, 2, 1, 100, 64), scale=0.4, cap=10.0, slopes=[0.1, 0.0])
    check(vfa, *prompt(7, 1, 2, 1, 100, 64), scale=0.02)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 1.0])
def test_scales_and_slopes_at_the_ends(vfa, d, cap):
    for N in (40, 500):
        check(vfa, *prompt(7, 1, 2, 1, N, d), scale=2.0 ** -64, cap=cap, slopes=[0.3, 2.0 ** 18])
        check(vfa, *prompt(7, 1, 2, 1, N, d), scale=2.0 ** -64, cap=cap, slopes=[-(2.0 ** 18), 2.0 ** 12], causal=False)
        check(vfa, *prompt(7, 1, 2, 1, N, d), scale=2.0 ** 16, cap=cap, slopes=[0.3, 0.0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", SCORES)
def test_long(vfa, d, cap, bias):
    """Rows of a longer prompt: first, last and some between."""
    N = 3001
    Q, K, V = prompt(2, 1, 4, 2, N, d, 6.0 if cap else 1.5)
    rows = torch.tensor([0, 1, 63, 64, 127, 128, 1000, 1500, 2047, 2048, 2999, 3000])
    kw = dict(cap=cap, slopes=[2.0 ** -h for h in range(1, 5)] if bias else None, rows=rows)
    check(vfa, Q, K, V, **kw)
    check(vfa, Q, K, V, causal=False, **kw)
    docs = vfa.row_ranges(ints([[0, 100, 1100, 1101, 2500, N]]), N)
    check(vfa, Q, K, V, ranges=docs.cpu(), **kw)


def test_capped_scores_at_both_ends(vfa):
    """All scores at -cap, all at +cap, and some of each: a row's max may be anywhere."""
    for cap in (20.0, 43.0, 50.0, 100.0):
        Q, K, V = prompt(3, 1, 2, 1, 300, 64)
        Q = Q.abs() * 8
        K = K.abs() * 8
        K[:, :, :150] *= -1
        check(vfa, Q, K, V, cap=cap)
        check(vfa, Q, -K, V, cap=cap)
        check(vfa, Q, -K.abs(), V, cap=cap)
        check(vfa, Q, K.abs(), V, cap=cap, slopes=[0.0, 1.0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("x", [math.nan, math.inf, -math.inf])
def test_special_values_stay_in_their_document(vfa, d, x):
    """NaN and infinities of a document, or of padding, reach no other one: those have the bits that they have without."""
    N, o = 500, [0, 100, 130, 131, 333, 450]
    Q, K, V = prompt(d, 1, 4, 2, N, d)
    ranges = vfa.row_ranges(ints([o]), N)
    clean, clean_l = vfa.masked_attn_fwd(Q.cuda(), K.cuda(), V.cuda(), ranges=ranges)
    for lo, hi in ((100, 130), (130, 131), (450, 500), (0, 100)):
        k, v, q = K.clone(), V.clone(), Q.clone()
        v[:, :, lo:hi, ::3] = x
        k[:, :, lo:hi] = x
        q[:, :, lo:hi] = x
        O, lse = vfa.masked_attn_fwd(q.cuda(), k.cuda(), v.cuda(), ranges=ranges)
        keep = torch.ones(N, dtype=torch.bool)
        keep[lo:hi] = False
        keep = keep.cuda()
        assert torch.equal(O[:, :, keep], clean[:, :, keep]) and torch.equal(lse[:, :, keep], clean_l[:, :, keep]), (lo, hi)


@pytest.mark.parametrize("d", [64, 128])
def test_special_values_behind_a_row(vfa, d):
    """Values that are not finite reach the rows that see their key, and no others: causal, prefixes, all."""
    N = 300
    Q, K, V = prompt(d, 1, 2, 1, N, d)
    for t, f, x in ((40, 3, math.inf), (41, 3, -math.inf), (70, 5, math.nan), (150, 7, math.inf), (290, 9, -math.inf), (290, 10, math.nan), (128, 11, math.inf)):
        V[:, :, t, f::32] = x
    check(vfa, Q, K, V)
    check(vfa, Q, K, V, ranges=vfa.row_ranges(ints([[0, 45, 200, N]]), N, prefix_lens=ints([[42, 20, 95]])).cpu())
    check(vfa, Q, K, V, ranges=vfa.row_ranges(ints([[0, 45, 200, N]]), N, causal=False).cpu(), cap=20.0)


def test_rows_behind_the_end_are_not_read(vfa):
    """The last tile's rest is nobody's: a prompt at the end of a larger tensor of NaN."""
    N, d = 77, 128
    big = [torch.full((4, 1, 2 * N, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    Q, K, V = prompt(5, 1, 1, 1, N, d)
    want = vfa.masked_attn_fwd(Q.cuda(), K.cuda(), V.cuda())
    views = []
    for b, x in zip(big, (Q, K, V)):
        v = b.view(-1)[: N * d].view(1, 1, N, d)
        v.copy_(x)
        views.append(v)
    got = vfa.masked_attn_fwd(*views)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_same_bits_and_outputs_given(vfa):
    Q, K, V = (x.cuda() for x in prompt(6, 2, 4, 2, 500, 128))
    O, lse = vfa.masked_attn_fwd(Q, K, V, score_cap=30.0)
    for _ in range(3):
        a, b = vfa.masked_attn_fwd(Q, K, V, score_cap=30.0)
        assert torch.equal(a, O) and torch.equal(b, lse)
    o, l = torch.full_like(Q, math.nan), torch.full((2, 4, 500), math.nan, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    r = vfa.masked_attn_fwd(Q, K, V, score_cap=30.0, out=o, lse=l, stream=s)
    x, y = vfa.masked_attn_fwd(Q, K, V, score_cap=30.0, stream=s)
    s.synchronize()
    assert r[0] is o and torch.equal(o, O) and torch.equal(l, lse) and torch.equal(x, O) and torch.equal(y, lse)
    assert vfa.masked_attn_fwd(Q, K, V, want_lse=False)[1] is None
    assert vfa.masked_attn_fwd(Q[:, :, :0], K[:, :, :0], V[:, :, :0])[0].shape == (2, 4, 0, 128)
    assert vfa.masked_attn_fwd(Q[:0], K[:0], V[:0])[0].shape == (0, 4, 500, 128)


# ---- the run of a server ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,cap,bias", [(128, 50.0, False), (64, 0.0, True), (128, 0.0, False)])
def test_prompt_then_steps(vfa, d, cap, bias):
    """Two prompts packed into one row, their rows into pages, then steps and drafts: what each new token gets is what the whole sequence in one prompt gives."""
    g = torch.Generator().manual_seed(d)
    Hq, H, page, lens, steps = 4, 2, 16, [150, 71], [1, 3, 1]
    total = [n + sum(steps) for n in lens]
    slopes = torch.tensor([0.5, 0.25, 0.1, 0.01], device="cuda") if bias else None
    full = [[torch.randn((h, n, d), generator=g).to(torch.bfloat16).cuda() for h in (Hq, H, H)] for n in total]
    cat = lambda i: torch.cat([full[b][i][:, : lens[b]] for b in range(2)], 1)[None].contiguous()
    ranges = vfa.row_ranges(ints([[0, 150, 221]]), 221)
    O, _ = vfa.masked_attn_fwd(cat(0), cat(1), cat(2), ranges=ranges, score_cap=cap, slopes=slopes)
    cache = vfa.kvp_cache(40, H, page, d)
    for t in cache:
        t.fill_(math.nan)
    table = torch.randperm(40, generator=g)[:24].int().reshape(2, 12).cuda()
    start = 0
    for b in range(2):
        vfa.kvp_append(cat(1)[:, :, start: start + lens[b]], cat(2)[:, :, start: start + lens[b]], cache, table[b: b + 1], 0, lens[b])
        start += lens[b]
    out = [[O[0, :, :150]], [O[0, :, 150:]]]
    now = list(lens)
    for n in steps:
        new = [x + n for x in now]
        q, k, v = (torch.stack([full[b][i][:, now[b]: new[b]] for b in range(2)]).contiguous() for i in range(3))
        vfa.kvp_append(k, v, cache, table, ints(now), ints(new))
        o, _ = vfa.kvp_decode_fwd(q, cache, table, ints(new), score_cap=cap, slopes=slopes)
        for b in range(2):
            out[b].append(o[b])
        now = new
    for b in range(2):
        n = total[b]
        key = torch.arange(n)
        for h in range(Hq):
            q, k, v = full[b][0][h].cpu(), full[b][1][h // 2].cpu(), full[b][2][h // 2].cpu()
            want = attend(q, k, v, key[None] <= key[:, None], (key[:, None] - key).abs().double(), cap, float(slopes[h]) if bias else None)
            got = torch.cat(out[b], 1)[h]
            compare(got, want[1], *want, (b, h))


def test_replayed(vfa):
    """A prompt and a step in one graph, replayed with new inputs, lengths and tables."""
    g = torch.Generator().manual_seed(0)
    B, Hq, H, N, d, page = 2, 8, 2, 200, 128, 16
    Q, K, V = (torch.zeros((B, h, N, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    q, k, v = (torch.zeros((B, h, 1, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    cache = vfa.kvp_cache(64, H, page, d)
    for t in cache:
        t.zero_()
    table, old, new, offsets = torch.zeros((B, 20), dtype=torch.int32, device="cuda"), ints([0, 0]), ints([1, 1]), ints([[0, 5, 200]] * 2)
    ranges = torch.zeros((B, N, 2), dtype=torch.int32, device="cuda")
    O, L, o, l = torch.empty_like(Q), torch.empty((B, Hq, N), device="cuda"), torch.empty_like(q), torch.empty((B, Hq, 1), device="cuda")
    ws = torch.empty(vfa.kvp_decode_workspace_bytes(B, Hq, 1, d, 3), dtype=torch.uint8, device="cuda")

    def work():
        vfa.row_ranges(offsets, N, out=ranges)
        vfa.masked_attn_fwd(Q, K, V, ranges=ranges, score_cap=30.0, out=O, lse=L)
        vfa.kvp_append(k, v, cache, table, old, new)
        vfa.kvp_decode_fwd(q, cache, table, new, n_splits=3, score_cap=30.0, workspace=ws, out=o, lse=l)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for rnd in range(3):
        for t in (Q, K, V, q, k, v, *cache):
            t.copy_(torch.randn(t.shape, generator=g))
        table.copy_(torch.randperm(64, generator=g)[:40].reshape(2, 20))
        n = [17 + 90 * rnd, 300 - 50 * rnd]
        old.copy_(torch.tensor(n))
        new.copy_(torch.tensor(n) + 1)
        offsets.copy_(torch.tensor([[0, 60 + rnd, 200 - rnd], [rnd, 128, 130]]))
        before = [t.clone() for t in cache]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in (O, L, o, l, *cache)]
        for t, x in zip(cache, before):
            t.copy_(x)
        for t in (O, L, o, l):
            t.fill_(math.nan)
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(seen, (O, L, o, l, *cache))), rnd
