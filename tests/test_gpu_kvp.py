"""The paged cache: rows written into pages, and the attention of the newest tokens over them, against 64 bits."""
import math

import pytest
import torch

from masked_util import HALF_BF16, attend, compare, paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vfa():
    import paper_2604_12798_amd as p
    p.lib()
    return p


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- append ----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,H,old,n", [(16, 2, [0, 5, 15, 16, 31], 1), (16, 3, [0, 7, 16], 5), (32, 1, [3, 100], 70), (64, 2, [0, 63, 64, 129], 64),
                                          (256, 2, [250, 0], 300), (16, 1, [1], 1025)])
def test_append(vfa, d, page, H, old, n):
    g = gen(d + page + n)
    B, new = len(old), [o + n for o in old]
    cap = max(new) + page
    _, _, pool, table = paged(g, new, H, d, page, cap, fill=3.0)
    K, V = (torch.randn((B, H, n, d), generator=g).to(torch.bfloat16) for _ in range(2))
    want = [p.clone() for p in pool]
    for b in range(B):
        for i in range(n):
            pg, r = int(table[b, (old[b] + i) // page]), (old[b] + i) % page
            want[0][pg, :, r], want[1][pg, :, r] = K[b, :, i], V[b, :, i]
    for lens in ((ints(old), ints(new)), None):
        if lens is None and len(set(old)) > 1:
            continue
        cache = tuple(p.cuda() for p in pool)
        out = vfa.kvp_append(K.cuda(), V.cuda(), cache, table.cuda(), *(lens or (old[0], new[0])))
        assert out is cache
        for got, w in zip(cache, want):
            assert torch.equal(got.cpu(), w)


def test_append_takes_slices_of_a_projection(vfa):
    g = gen(1)
    x = torch.randn((3, 20, 2 + 2 * 2, 128), generator=g).to(torch.bfloat16).cuda()   # [B, N, Hq + 2 Hkv, d]
    K, V = x[:, :, 2:4].transpose(1, 2), x[:, :, 4:].transpose(1, 2)
    _, _, pool, table = paged(g, [25, 30, 20], 2, 128, 16, 48)
    a, b = (tuple(p.cuda() for p in pool) for _ in range(2))
    old, new = ints([5, 10, 0]), ints([25, 30, 20])
    vfa.kvp_append(K, V, a, table.cuda(), old, new)
    vfa.kvp_append(K.contiguous(), V.contiguous(), b, table.cuda(), old, new)
    for s, t in zip(a, b):
        assert torch.equal(s.view(torch.int16), t.view(torch.int16))


def test_append_leaves_out_holes_and_what_is_past_the_ends(vfa):
    """Entries outside the pool take nothing; lengths are clamped to the table's capacity; old >= new writes nothing; rows past n_in do not exist."""
    g = gen(2)
    H, d, page, M, P = 2, 64, 16, 4, 9
    pool = [torch.full((P, H, page, d), 3.0, dtype=torch.bfloat16) for _ in range(2)]
    table = torch.tensor([[0, -1, 1, P], [2, 3, 2 ** 31 - 1, -2 ** 31], [4, 5, 6, 7]], dtype=torch.int32)
    n = 40
    K, V = (torch.randn((3, H, n, d), generator=g).to(torch.bfloat16) for _ in range(2))
    for old, new in (([3, 0, 30], [43, 40, 70]), ([-5, 20, 10], [35, 10, 2 ** 31 - 1]), ([50, 2 ** 31 - 1, -2 ** 31], [90, 2 ** 31 - 1, 3]), ([0, 0, 0], [64, 64, 64])):
        want = [p.clone() for p in pool]
        for b in range(3):
            o = min(max(old[b], 0), M * page)
            for t in range(o, min(new[b], M * page, o + n)):
                pg = int(table[b, t // page])
                if 0 <= pg < P:
                    want[0][pg, :, t % page], want[1][pg, :, t % page] = K[b, :, t - o], V[b, :, t - o]
        cache = tuple(p.cuda() for p in pool)
        vfa.kvp_append(K.cuda(), V.cuda(), cache, table.cuda(), ints(old), ints(new))
        for got, w in zip(cache, want):
            assert torch.equal(got.cpu(), w), (old, new)


def test_append_of_nothing(vfa):
    cache = vfa.kvp_cache(2, 2, 16, 64)
    for t in cache:
        t.fill_(1)
    table = ints([[0, 1]])
    one = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    vfa.kvp_append(one[:, :, :0], one[:, :, :0], cache, table, 3, 3)
    vfa.kvp_append(one, one, cache, table, 3, 3)
    vfa.kvp_append(one[:0], one[:0], cache, table[:0], ints([]), ints([]))
    vfa.kvp_append(one, one, tuple(t[:0] for t in cache), table, 0, 1)
    vfa.kvp_append(one, one, cache, ints([[]]), ints([0]), ints([1]))
    assert all((t == 1).all() for t in cache)


# ---- decode ----------------------------------------------------------------------------------------------------------------------

def check_decode(vfa, g, lens, Hq, Hkv, d, page, n_q=1, cap=0.0, slopes=None, n_splits=None, number=False, holes=(), spoil=None, sharp=1.5, scale=None, slack=37):
    rows, there, pool, table = paged(g, lens, Hkv, d, page, max(lens) + slack, holes=holes)
    B, gq = len(lens), Hq // Hkv
    q = (sharp * torch.randn((B, Hq, n_q, d), generator=g)).to(torch.bfloat16)
    if spoil:
        spoil(q, rows, pool, table)
    s = None if slopes is None else torch.tensor(slopes, dtype=torch.float32)
    dev = dict(score_cap=cap, slopes=None if s is None else s.cuda(), n_splits=n_splits, **({} if scale is None else dict(softmax_scale=scale)))
    O, lse = vfa.kvp_decode_fwd(q.cuda(), tuple(p.cuda() for p in pool), table.cuda(), lens[0] if number else ints(lens), **dev)
    exactly = gq * n_q <= 16
    for b, n in enumerate(lens):
        pos = torch.arange(n - n_q, n)[:, None]
        key = torch.arange(n)[None]
        seen = (key <= pos) & there[b][None]
        away = (pos - key).abs().double()
        for h in range(Hq):
            k, v = rows[b][0][h // gq], rows[b][1][h // gq]
            want = attend(q[b, h], torch.where(there[b][:, None], k, 0), torch.where(there[b][:, None], v, 0), seen, away, cap,
                          None if s is None else float(s[h]), scale, weights=2.0 ** -15 if exactly else HALF_BF16)
            compare(O[b, h], lse[b, h], *want, (b, h, n))
    return O, lse


HEADS = [(4, 2), (8, 1), (3, 3), (16, 1), (20, 1), (32, 1)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_decode(vfa, d, page, Hq, Hkv):
    g = gen(d * page + Hq)
    check_decode(vfa, g, [1, 15, 16, 17, 63, 64, 65, 130, 300, 700], Hq, Hkv, d, page)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_splits", [1, 2, 3, 7, 40])
@pytest.mark.parametrize("number", [False, True])
def test_decode_ranges(vfa, d, n_splits, number):
    lens = [1000] * 3 if number else [1000, 0, 3, 129, 640]
    check_decode(vfa, gen(n_splits), lens, 4, 2, d, 16, n_splits=n_splits, number=number)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_splits", [1, 3])
@pytest.mark.parametrize("Hq,Hkv,n_q", [(2, 2, 2), (4, 2, 4), (4, 2, 8), (8, 2, 5), (4, 2, 16), (4, 2, 17), (12, 4, 40), (32, 1, 3), (2, 2, 100)])
def test_decode_newest_tokens(vfa, d, n_splits, Hq, Hkv, n_q):
    check_decode(vfa, gen(n_q), [1, n_q, 64, 66, 128, 333], Hq, Hkv, d, 32, n_q=n_q, n_splits=n_splits)


SLOPES = [0.5, 0.011, 1.7, 0.0, -0.003, 0.08, 0.2, 0.9]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", [(30.0, False), (0.0, True), (50.0, True), (5.0, False), (1000.0, False), (0.001, True)])
@pytest.mark.parametrize("n_q,n_splits", [(1, None), (1, 3), (5, 2), (20, 1)])
def test_decode_scores(vfa, d, cap, bias, n_q, n_splits):
    check_decode(vfa, gen(int(cap) + n_q), [1, 40, 64, 200, 777], 8, 2, d, 16, n_q=n_q, cap=cap, slopes=SLOPES if bias else None, n_splits=n_splits, sharp=6.0)


def test_decode_scale(vfa):
    check_decode(vfa, gen(3), [100, 200], 8, 2, 64, 16, cap=20.0, slopes=SLOPES, scale=0.3)
    check_decode(vfa, gen(3), [100, 200], 8, 2, 64, 16, scale=0.01)
    for cap in (0.0, 1.0):
        check_decode(vfa, gen(3), [100, 200], 8, 2, 64, 16, cap=cap, slopes=SLOPES[:7] + [2.0 ** 20], scale=2.0 ** -64)
        check_decode(vfa, gen(3), [100, 200], 8, 2, 64, 16, cap=cap, slopes=SLOPES, scale=2.0 ** 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_q,n_splits", [(1, 1), (1, 4), (6, 2), (30, 1)])
def test_decode_holes(vfa, d, page, n_q, n_splits):
    """Pages that are not there: at the start, in the middle, the newest one, all of them."""
    lens = [5 * page + 3, 9 * page, 2 * page, 7 * page + page // 2]
    holes = {(0, 0), (0, 3), (1, 4), (1, 5), (1, 8), (2, 0), (2, 1), (3, 7)}
    check_decode(vfa, gen(page + n_q), lens, 4, 2, d, page, n_q=n_q, n_splits=n_splits, holes=holes, slopes=[0.1, 0.2, 0.0, 0.3])


def test_decode_does_not_see_what_is_not_there(vfa):
    """All of the pool but the sequences' rows is NaN in every test here; infinities are the same."""
    g = gen(5)
    rows, there, pool, table = paged(g, [70, 130], 2, 128, 64, 192, fill=math.inf)
    q = torch.randn((2, 4, 2, 128), generator=g).to(torch.bfloat16).cuda()
    O, lse = vfa.kvp_decode_fwd(q, tuple(p.cuda() for p in pool), table.cuda(), ints([70, 130]))
    assert torch.isfinite(O).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n_q", [(4, 2, 6), (4, 2, 10), (4, 2, 40)])
@pytest.mark.parametrize("n_splits", [1, 2])
def test_decode_special_values_of_newest_tokens(vfa, d, Hq, Hkv, n_q, n_splits):
    """Infinities and NaN among the values (and NaN among the keys) of drafts reach those rows that see them, and no others."""
    def spoil(q, rows, pool, table):
        for b, n in enumerate([64, 130, 200]):
            for back, kv, x in ((1, 1, math.nan), (2, 1, math.inf), (3, 1, -math.inf), (4, 1, math.inf), (1, 0, math.nan)):
                t = n - back
                for f in range(0, d, 5) if back != 4 else range(3, d, 11):
                    rows[b][kv][:, t, f] = x
                    pool[kv][int(table[b, t // 32]), :, t % 32, f] = x
    g = gen(d + n_q)
    lens = [64, 130, 200]
    rows, there, pool, table = paged(g, lens, Hkv, d, 32, 230)
    q = torch.randn((3, Hq, n_q, d), generator=g).to(torch.bfloat16)
    spoil(q, rows, pool, table)
    O, lse = vfa.kvp_decode_fwd(q.cuda(), tuple(p.cuda() for p in pool), table.cuda(), ints(lens), n_splits=n_splits)
    for b, n in enumerate(lens):
        pos, key = torch.arange(n - n_q, n)[:, None], torch.arange(n)[None]
        for h in range(Hq):
            k, v = rows[b][0][h * Hkv // Hq], rows[b][1][h * Hkv // Hq]
            sub = slice(0, n_q - 1)  # (the last row's scores are NaN)
            want = attend(q[b, h, sub], torch.where(k.isnan(), 0, k), v, (key <= pos)[sub], (pos - key)[sub].abs().double(), 0.0, None,
                          weights=2.0 ** -15 if Hq // Hkv * n_q <= 16 else HALF_BF16)
            compare(O[b, h, sub], lse[b, h, sub], *want, (b, h))
            assert O[b, h, -1].isnan().all()


def test_decode_infinite_value_that_all_see(vfa):
    """An infinity among the values of an old key is one in every row, also where its weight has 16 bits or fewer (one key: the weight is 1)."""
    for n in (1, 64, 200):
        g = gen(n)
        rows, there, pool, table = paged(g, [n], 1, 128, 16, n)
        pool[1][int(table[0, 0]), 0, 0, 3], pool[1][int(table[0, 0]), 0, 0, 4] = math.inf, -math.inf
        q = torch.randn((1, 4, 128), generator=g).to(torch.bfloat16).cuda()
        O, _ = vfa.kvp_decode_fwd(q, tuple(p.cuda() for p in pool), table.cuda(), n, n_splits=1)
        assert (O[0, :, 3] == math.inf).all() and (O[0, :, 4] == -math.inf).all() and torch.isfinite(O[0, :, 5:]).all()


def test_decode_many_sequences(vfa):
    """More entries than ranges are dealt for, and one that reads the same pages as another."""
    g = gen(9)
    lens = [int(x) for x in torch.randint(0, 200, (300,), generator=g)]
    check_decode(vfa, g, lens, 2, 1, 64, 16, n_splits=2)
    rows, there, pool, table = paged(g, [150], 2, 128, 16, 160)
    q = torch.randn((1, 4, 128), generator=g).to(torch.bfloat16)
    cache = tuple(p.cuda() for p in pool)
    one, l1 = vfa.kvp_decode_fwd(q.cuda(), cache, table.cuda(), 150, n_splits=1)
    both, l2 = vfa.kvp_decode_fwd(q.repeat(2, 1, 1).cuda(), cache, table.repeat(2, 1).cuda(), ints([150, 150]), n_splits=1)
    assert torch.equal(both[0], one[0]) and torch.equal(both[1], one[0]) and torch.equal(l2[1], l1[0])


def test_decode_of_nothing(vfa):
    cache = vfa.kvp_cache(0, 2, 16, 64)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for table, lens in ((ints([[], []]), 0), (ints([[0, 1], [2, 3]]), 20), (ints([[], []]), ints([3, 4]))):
        for ns in (1, 3):
            O, lse = vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=ns)
            assert (O == 0).all() and (lse == -math.inf).all()
    O, lse = vfa.kvp_decode_fwd(q[:, :, None][:, :, :0], cache, ints([[], []]), 0)
    assert O.shape == (2, 4, 0, 64)
    O, lse = vfa.kvp_decode_fwd(q[:0], cache, ints([[], []])[:0], ints([]))
    assert O.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_decode_takes_outputs_and_streams(vfa):
    g = gen(11)
    rows, there, pool, table = paged(g, [500, 300], 2, 128, 16, 512)
    cache, table = tuple(p.cuda() for p in pool), table.cuda()
    q = torch.randn((2, 8, 3, 128), generator=g).to(torch.bfloat16).cuda()
    lens = ints([500, 300])
    O, lse = vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=3)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, b = vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=3, stream=s)
    ws = torch.empty(vfa.kvp_decode_workspace_bytes(2, 8, 3, 128, 3), dtype=torch.uint8, device="cuda")
    o, l = torch.full_like(q, math.nan), torch.full((2, 8, 3), math.nan, device="cuda")
    torch.cuda.synchronize()
    c, e = vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=3, workspace=ws, out=o, lse=l, stream=s)
    s.synchronize()
    assert c is o and e is l
    for x, y in ((a, O), (b, lse), (o, O), (l, lse)):
        assert torch.equal(x, y)
    none = vfa.kvp_decode_fwd(q, cache, table, lens, n_splits=3, want_lse=False)
    assert none[1] is None and torch.equal(none[0], O)


def test_pages_past_four_gigabytes(vfa):
    """A pool of 6 GiB each: offsets of pages do not fit 32 bits."""
    H, d, page, n = 8, 128, 256, 300
    P = (6 << 30) // (H * d * page * 2)
    K, V = (torch.empty((P, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = ints([[P - 1, P // 2 + 3], [5, P - 7]])
    g = gen(12)
    k, v = (torch.randn((2, H, n, d), generator=g).to(torch.bfloat16) for _ in range(2))
    vfa.kvp_append(k.cuda(), v.cuda(), (K, V), table, 0, n)
    for b in range(2):
        for t in range(2):
            at, end = t * page, min(n, t * page + page)
            assert torch.equal(K[int(table[b, t]), :, : end - at].cpu(), k[b, :, at:end])
    q = torch.randn((2, 16, d), generator=g).to(torch.bfloat16)
    O, lse = vfa.kvp_decode_fwd(q.cuda(), (K, V), table, n)
    for b in range(2):
        for h in range(16):
            want = attend(q[b, h][None], k[b, h // 2], v[b, h // 2], torch.ones((1, n), dtype=torch.bool), None, 0.0, None, weights=2.0 ** -15)
            compare(O[b, h][None], lse[b, h][None], *want, (b, h))
