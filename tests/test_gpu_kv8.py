"""The 8-bit cache on the GPU: writing (codes and scales bit for bit), reading back (bit for bit), attention of one and more new tokens against
64 bits, and a serving loop of all of them."""
import math

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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(shape, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * size
    x[..., : shape[-1] // 8] *= 7
    return x.to(torch.bfloat16)


def same_cache(cache, want, new):
    """Tokens below `new` of each sequence, and the scales of their blocks."""
    codes, exp = ref.unpack(cache)
    for side in range(2):
        for b, n in enumerate(new):
            assert ref.same_codes(codes[side][b, :, :n], want.codes[side][b, :, :n]), (side, b)
            t = -(-n // 64)
            assert torch.equal(exp[side][b, :, :t], want.exp[side][b, :, :t]), (side, b)


# ---- writing ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 300])
def test_first_rows(vfa, d, n):
    B, H, cap = 2, 3, 320
    K, V = rows((B, H, n, d), n), rows((B, H, n, d), n + 1, 0.01)
    cache = vfa.kv8_cache(B, H, cap, d)
    for t in cache:
        t.fill_(0x55)
    vfa.kv8_append(K.cuda(), V.cuda(), cache, 0, n)
    want = ref.Cache(B, H, cap, d)
    want.append(K, V, [0] * B, [n] * B)
    same_cache(cache, want, [n] * B)
    codes, exp = ref.unpack(cache)
    for side in range(2):  # what lies behind is as it was
        assert (codes[side][:, :, n:] == 0x55).all() and (exp[side][:, :, -(-n // 64):] == 0x55 - 127).all()


@pytest.mark.parametrize("d", [64, 128])
def test_growing_with_larger_and_smaller_rows(vfa, d):
    """Token by token and by more, over the ends of blocks; a row that needs a larger scale has the block coded again, and tokens behind a rewound
    length are written anew."""
    B, H, cap = 2, 2, 256
    cache, want = vfa.kv8_cache(B, H, cap, d), ref.Cache(B, H, cap, d)
    n, size = 0, [1, 1, 30, 0.01, 4, 1e4, 1, 1e-3, 1e5, 2, 2, 1e6, 1]
    for i, step in enumerate((1, 1, 5, 50, 7, 1, 63, 64, 1, -20, 3, 17, 2)):
        if step < 0:
            n += step
            continue
        K, V = rows((B, H, step, d), 100 + i, size[i]), rows((B, H, step, d), 200 + i, size[-1 - i])
        vfa.kv8_append(K.cuda(), V.cuda(), cache, n, n + step)
        want.append(K, V, [n] * B, [n + step] * B)
        n += step
        same_cache(cache, want, [n] * B)


def test_recoding_into_subnormals(vfa):
    """Every code in a block whose scale grows by 2^0 to 2^40."""
    for grow in (0, 1, 2, 3, 7, 9, 12, 18, 40):
        codes = torch.arange(256, dtype=torch.uint8).repeat(32).reshape(1, 1, 64, 128)
        want = ref.Cache(1, 1, 64, 128)
        want.codes = [codes.clone(), codes.flip(2).contiguous()]
        want.exp = [torch.full((1, 1, 1), -3, dtype=torch.int32) for _ in range(2)]
        cache = ref.pack(want)
        x = torch.full((1, 1, 1, 128), 448 * 2.0 ** (grow - 3)).to(torch.bfloat16)
        vfa.kv8_append(x.cuda(), x.cuda(), cache, 63, 64)
        want.append(x, x, [63], [64])
        same_cache(cache, want, [64])


def test_every_bf16(vfa):
    """All finite values of bf16, 64 neighbours to a row, so that a block spans a few binades; then each alone with the largest of its block."""
    bits = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.where(bits.isfinite(), bits, torch.zeros_like(bits)).reshape(1, 1, 512, 128)
    for y in (x, x.reshape(64, 8, 128).transpose(0, 1).reshape(1, 1, 512, 128).contiguous()):
        cache, want = vfa.kv8_cache(1, 1, 512, 128), ref.Cache(1, 1, 512, 128)
        vfa.kv8_append(y.cuda(), y.cuda(), cache, 0, 512)
        want.append(y, y, [0], [512])
        same_cache(cache, want, [512])


def test_zeros_infinities_nan(vfa):
    K = rows((1, 2, 130, 64), 5)
    K[0, 0, 3, 7], K[0, 0, 4, 7], K[0, 0, 70, 0], K[0, 1, 129, 63] = math.inf, -math.inf, math.nan, math.nan
    V = torch.zeros((1, 2, 130, 64), dtype=torch.bfloat16)
    V[0, 0, :64] = math.inf
    V[0, 1, :64] = math.nan
    V[0, 1, 128] = -0.0
    cache, want = vfa.kv8_cache(1, 2, 192, 64), ref.Cache(1, 2, 192, 64)
    vfa.kv8_append(K.cuda(), V.cuda(), cache, 0, 130)
    want.append(K, V, [0], [130])
    same_cache(cache, want, [130])
    assert int(cache[3][0, 0, 1]) == ref.E_MIN + 127


@pytest.mark.parametrize("d", [64, 128])
def test_ragged_batch(vfa, d):
    """Lengths of their own, among them empty, full, reversed, beyond the capacity and with more rows than were given."""
    B, H, cap, n_in = 8, 2, 192, 70
    old = [0, 0, 63, 64, 100, 150, -5, 192]
    new = [0, 70, 64, 134, 60, 500, 3, 400]
    o = [min(max(x, 0), cap) for x in old]
    n = [min(min(y, cap), x + n_in) for x, y in zip(o, new)]
    want = ref.random_cache(B, H, cap, d, 3)
    cache = ref.pack(want)
    K, V = rows((B, H, n_in, d), 1, 3), rows((B, H, n_in, d), 2, 0.1)
    vfa.kv8_append(K.cuda(), V.cuda(), cache, ints(old), ints(new))
    want.append(K, V, o, n)
    same_cache(cache, want, [cap] * B)  # everything else is as it was


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H", [1, 3, 8])
def test_one_row_each(vfa, d, H):
    """One new token for each sequence, several times: at a block's beginning, middle and end, none, at the capacity, rows that need a larger scale in
    some heads only, of keys or of values."""
    cap = 192
    old = [0, 1, 3, 62, 63, 64, 100, 127, 128, 191, 192, 50, -4]
    new = [o + 1 for o in old]
    new[11], new[6] = 50, 5000
    B = len(old)
    o = [min(max(x, 0), cap) for x in old]
    n = [min(min(y, cap), x + 1) for x, y in zip(o, new)]
    want = ref.random_cache(B, H, cap, d, 3)
    cache = ref.pack(want)
    for i in range(4):
        K, V = rows((B, H, 1, d), 10 + i), rows((B, H, 1, d), 20 + i)
        grow = torch.randint(0, 12, (2, B, H, 1, 1), generator=torch.Generator().manual_seed(i))
        K, V = (K * 2.0 ** grow[0]).to(torch.bfloat16), (V * 2.0 ** grow[1]).to(torch.bfloat16)
        vfa.kv8_append(K.cuda(), V.cuda(), cache, ints(old), ints(new))
        want.append(K, V, o, n)
        same_cache(cache, want, [cap] * B)


def test_strides(vfa):
    """Keys and values as slices of one projection, a head axis of stride zero, a batch run backwards through memory."""
    B, H, n, d = 2, 3, 37, 128
    x = rows((B, n, 2 * H, d), 8).cuda()
    K, V = x[:, :, :H].transpose(1, 2), x[:, :, H:].transpose(1, 2)
    one = x[:, :, :1].transpose(1, 2).expand(B, H, n, d)
    for k, v in ((K, V), (one, K), (V.contiguous(), one)):
        cache, want = vfa.kv8_cache(B, H, 64, d), ref.Cache(B, H, 64, d)
        vfa.kv8_append(k, v, cache, 5, 5 + n)  # (rows 0 to 4 hold anything: only the new ones are looked at)
        cache2 = vfa.kv8_cache(B, H, 64, d)
        for a, c in zip(cache2, cache):
            a.copy_(c)
        vfa.kv8_append(k, v, cache2, 0, n)
        want.append(k.cpu(), v.cpu(), [0] * B, [n] * B)
        same_cache(cache2, want, [n] * B)


def test_more_rows_than_fit(vfa):
    """As many rows as an int counts (all of them one row), of which few are taken; lengths at the ends of their type."""
    B, H, cap, d = 5, 2, 192, 64
    old, new = [100, 0, 191, 2 ** 31 - 1, -2 ** 31], [101, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31]
    one = rows((B, H, 1, d), 6)
    x = one.cuda().expand(B, H, 2 ** 31 - 1, d)
    want = ref.random_cache(B, H, cap, d, 5)
    cache = ref.pack(want)
    vfa.kv8_append(x, x, cache, ints(old), ints(new))
    few = one.expand(B, H, cap, d)
    want.append(few, few, [100, 0, 191, 192, 0], [101, 192, 192, 192, 0])
    same_cache(cache, want, [cap] * B)


def test_empty(vfa):
    """No sequences, no new rows, no capacity."""
    for B, n, cap in ((0, 3, 64), (2, 0, 64), (2, 0, 0)):
        cache = vfa.kv8_cache(B, 2, cap, 64)
        x = torch.zeros((B, 2, n, 64), dtype=torch.bfloat16, device="cuda")
        vfa.kv8_append(x, x, cache, 0, min(n, cap))
        vfa.kv8_append(x, x, cache, ints([0] * B), ints([5] * B))
        assert vfa.kv8_read(cache, 0)[0].shape == (B, 2, 0, 64)
        q = torch.zeros((B, 4, 3, 64), dtype=torch.bfloat16, device="cuda")
        for lens in (0, ints([0] * B)):
            for ns in (None, 1, 4):
                O, L = vfa.kv8_decode_fwd(q, cache, lens, n_splits=ns)
                assert (O == 0).all() and L.isneginf().all()
        assert vfa.kv8_decode_fwd(q[:, :, :0].contiguous(), cache, 0)[0].shape == (B, 4, 0, 64)


# ---- reading back ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 192])
def test_read(vfa, d, n):
    B, H, cap = 4, 2, 192
    want = ref.random_cache(B, H, cap, d, n)
    want.codes[0][0, 0, 0, 0] = 127
    lens = [n, 0, max(n - 1, 0), 500]
    out = [torch.full((B, H, n, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    got = vfa.kv8_read(ref.pack(want), n, seq_lens=ints(lens), out=out)
    for x, v in zip(got, want.values()):
        for b in range(B):
            m = min(lens[b], n)
            assert torch.equal(x[b, :, :m].cpu().nan_to_num(7.0), v[b, :, :m].to(torch.bfloat16).nan_to_num(7.0))
            assert (x[b, :, m:] == 0).all()
    again = vfa.kv8_read(ref.pack(want), n, seq_lens=n)
    assert torch.equal(again[1][3], got[1][3])


def test_read_extremes(vfa):
    """Every code at the smallest, middle and largest exponents."""
    want = ref.Cache(1, 1, 192, 128)
    codes = torch.arange(256, dtype=torch.uint8).repeat(96).reshape(1, 1, 192, 128)
    want.codes = [codes, codes.clone()]
    want.exp = [torch.tensor([[[ref.E_MIN, -9, 120]]], dtype=torch.int32) for _ in range(2)]
    for x, v in zip(vfa.kv8_read(ref.pack(want), 192), want.values()):
        assert torch.equal(x.cpu().nan_to_num(7.0, 8.0, 9.0), v.to(torch.bfloat16).nan_to_num(7.0, 8.0, 9.0))


# ---- attention -------------------------------------------------------------------------------------------------------------------

def run_decode(vfa, B, Hq, Hkv, cap, d, n_q, lens, n_splits, seed=0, uniform=False, q_size=1.5, **kw):
    c = ref.random_cache(B, Hkv, cap, d, seed)
    q = rows((B, Hq, n_q, d), seed + 1, q_size / 4).cuda()
    O = torch.full_like(q, math.nan)
    L = torch.full(q.shape[:3], math.nan, device="cuda")
    vfa.kv8_decode_fwd(q, ref.pack(c), lens[0] if uniform else ints(lens), n_splits=n_splits, out=O, lse=L, **kw)
    want = ref.attend(q, c.values(), [min(max(n, 0), cap) for n in lens], **({"scale": kw["softmax_scale"]} if "softmax_scale" in kw else {}))
    ref.check(O, L, want, (B, Hq, Hkv, cap, d, n_q, lens, n_splits))
    return O, L


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 4, 7, 16, 17, 32])
@pytest.mark.parametrize("n_splits", [1, 3, 24])
def test_decode_lengths(vfa, d, g, n_splits):
    lens = [0, 1, 63, 64, 65, 300, 512, 700, -3]
    run_decode(vfa, len(lens), 2 * g, 2, 512, d, 1, lens, n_splits, seed=g)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,n_q", [(1, 2), (1, 32), (4, 4), (4, 5), (8, 4), (3, 10), (16, 2), (5, 6)])
@pytest.mark.parametrize("n_splits", [1, 4])
def test_several_new_tokens(vfa, d, g, n_q, n_splits):
    """Among them sequences shorter than the number of new tokens, whose first ones see nothing, and new tokens on both sides of a block's end."""
    lens = [0, 1, n_q - 1, n_q, 64, 65, 64 + n_q // 2, 200]
    run_decode(vfa, len(lens), 2 * g, 2, 256, d, n_q, lens, n_splits, seed=n_q)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,n_q", [(4, 9), (4, 16), (1, 100), (7, 13), (32, 3), (3, 65), (20, 2), (8, 150)])
@pytest.mark.parametrize("n_splits", [None, 1, 3])
def test_pieces_of_a_prompt(vfa, d, g, n_q, n_splits):
    """More rows than one workgroup has: groups of whole tokens, a last group with fewer, tokens that see nothing, ranges that some groups have not."""
    lens = [0, 1, n_q - 1, n_q, n_q + 1, 64, 129, 192, 250]
    run_decode(vfa, len(lens), g, 1, 256, d, n_q, lens, n_splits, seed=n_q)
    run_decode(vfa, 1, 2 * g, 2, 1024, d, n_q, [1000], n_splits, seed=n_q)
    run_decode(vfa, 2, g, 1, 1024, d, n_q, [1000, 1000], n_splits, seed=n_q, uniform=True)


def test_pieces_of_many_sequences(vfa):
    """Batches above those whose ranges are dealt out."""
    run_decode(vfa, 260, 4, 1, 128, 64, 10, [(37 * b) % 129 for b in range(260)], 2, seed=1)


def test_a_prompt_in_pieces(vfa):
    """A prompt of 300 tokens written and attended to 70 at a time, against the causal pass over what the cache stands for."""
    B, Hq, H, d, N = 2, 8, 2, 128, 300
    K, V = rows((B, H, N, d), 50).cuda(), rows((B, H, N, d), 51).cuda()
    Q = rows((B, Hq, N, d), 52, 0.4).cuda()
    cache, got = vfa.kv8_cache(B, H, N, d), []
    for a in range(0, N, 70):
        b = min(N, a + 70)
        vfa.kv8_append(K[:, :, a:b], V[:, :, a:b], cache, a, b)
        got.append(vfa.kv8_decode_fwd(Q[:, :, a:b].contiguous(), cache, b))
    # (pieces that end inside a block see it under the scale that it has then; a second pass sees all as they are at the end)
    got = [vfa.kv8_decode_fwd(Q[:, :, a: a + 70].contiguous(), cache, ints([min(N, a + 70)] * B)) for a in range(0, N, 70)]
    O, L = torch.cat([o for o, _ in got], 2), torch.cat([l for _, l in got], 2)
    Kr, Vr = vfa.kv8_read(cache, N)
    want = ref.attend(Q, [Kr.double().cpu(), Vr.double().cpu()], [N] * B)
    ref.check(O, L, want)
    O2, L2 = vfa.vfa_attn_fwd(Q, Kr, Vr)
    assert (L - L2).abs().max() < 2e-3


@pytest.mark.parametrize("n", [0, 1, 64, 1000])
@pytest.mark.parametrize("n_splits", [None, 1, 5])
def test_one_length_for_all(vfa, n, n_splits):
    run_decode(vfa, 2, 8, 2, 1024, 128, 1, [n, n], n_splits, uniform=True, seed=n)
    run_decode(vfa, 2, 8, 2, 1024, 64, 3, [n, n], n_splits, uniform=True, seed=n)


@pytest.mark.parametrize("d,g,n_q", [(64, 3, 1), (64, 5, 5), (128, 4, 1), (128, 6, 4)])
@pytest.mark.parametrize("n_splits", [1, 2, 9])
def test_long_ranges(vfa, d, g, n_q, n_splits):
    """Ranges of many tiles for each wave, of four waves and of eight (64-wide heads in one range)."""
    run_decode(vfa, 3, 2 * g, 2, 4096, d, n_q, [4096, 1025, 3001], n_splits, seed=d + g)
    run_decode(vfa, 2, g, 1, 2048, d, n_q, [2011, 2011], n_splits, seed=d + g, uniform=True)


@pytest.mark.parametrize("B,n_splits", [(70, 2), (256, 3), (300, 2), (300, 1), (5000, None)])
def test_many_sequences(vfa, B, n_splits):
    """Batches whose ranges are dealt out, and batches above that."""
    run_decode(vfa, B, 4, 1, 320, 64, 1, [(37 * b) % 321 for b in range(B)], n_splits, seed=B)


def test_scale_and_large_scores(vfa):
    run_decode(vfa, 2, 4, 2, 256, 128, 1, [256, 100], 2, softmax_scale=0.5)
    run_decode(vfa, 2, 4, 2, 256, 128, 2, [256, 100], 2, q_size=20.0)


@pytest.mark.parametrize("up", [-90, -30, 30, 80])
def test_scales_of_any_size(vfa, up):
    """Keys 2^up times as large under a softmax scale as much smaller, and values 2^up times as large, bit for bit."""
    B, H, cap, d = 3, 2, 320, 128
    lens = ints([320, 63, 130])
    q = rows((B, 8, 2, d), 2, 0.4).cuda()
    c = ref.random_cache(B, H, cap, d, 1)
    O, L = vfa.kv8_decode_fwd(q, ref.pack(c), lens, n_splits=2, softmax_scale=2.0 ** -4)
    c.exp = [e + up for e in c.exp]
    O2, L2 = vfa.kv8_decode_fwd(q, ref.pack(c), lens, n_splits=2, softmax_scale=2.0 ** (-4 - up))
    assert torch.equal(L, L2) and torch.equal(O.double() * 2.0 ** up, O2.double())


def test_nothing_behind_the_end_is_seen(vfa):
    """NaN codes and scales of any kind behind a sequence's end, in its last block and beyond."""
    B, H, cap, d = 3, 2, 256, 128
    lens = [1, 70, 190]
    c = ref.random_cache(B, H, cap, d, 1)
    q = rows((B, 8, 2, d), 2, 0.4).cuda()
    clean = vfa.kv8_decode_fwd(q, ref.pack(c), ints(lens), n_splits=2)
    for side in range(2):
        for b, n in enumerate(lens):
            c.codes[side][b, :, n:] = 0x7f
            c.exp[side][b, :, -(-n // 64):] = 128
    dirty = vfa.kv8_decode_fwd(q, ref.pack(c), ints(lens), n_splits=2)
    assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1], dirty[1])


@pytest.mark.parametrize("d,g,n_q", [(64, 2, 4), (128, 6, 4), (64, 5, 11), (128, 3, 30)])
def test_nan_of_a_draft_reaches_those_who_see_it(vfa, d, g, n_q):
    """Keys and values that are NaN from the second and third of the last four new tokens: the tokens before them are clean."""
    B, H, cap = 2, 1, 192
    lens = [66, 140]
    for side in range(2):
        c = ref.random_cache(B, H, cap, d, 7)
        for b, n in enumerate(lens):
            c.codes[side][b, :, n - 3, 5] = 0x7f
            c.codes[side][b, :, n - 2, d - 1] = 0xff
        q = rows((B, g, n_q, d), 8, 0.4).cuda()
        for ns in (1, 2):
            O, L = vfa.kv8_decode_fwd(q, ref.pack(c), ints(lens), n_splits=ns)
            want = ref.attend(q, c.values(), lens)
            assert not want[0][:, :, : n_q - 3].isnan().any() and want[0][:, :, n_q - 3:].isnan().any()
            ref.check(O, L, want, (side, ns))


def test_offsets_past_32_bits(vfa):
    """Sequences that begin beyond 2^31 bytes of codes."""
    B, H, cap, d = 3, 8, 1 << 20, 128
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GiB")
    cache = vfa.kv8_cache(B, H, cap, d)
    n, far = 100, cap - 130
    K, V = rows((B, H, n, d), 1), rows((B, H, n, d), 2)
    vfa.kv8_append(K.cuda(), V.cuda(), cache, 0, n)
    small = vfa.kv8_cache(B, H, 128, d)
    vfa.kv8_append(K.cuda(), V.cuda(), small, 0, n)
    q = rows((B, 16, 1, d), 3).cuda()
    a, b = vfa.kv8_decode_fwd(q, cache, ints([n] * B), n_splits=2), vfa.kv8_decode_fwd(q, small, ints([n] * B), n_splits=2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    vfa.kv8_append(K.cuda(), V.cuda(), cache, ints([far] * B), ints([far + n] * B))
    t0 = far // 64
    want = ref.Cache(B, H, 256, d)
    want.append(K, V, [far % 64] * B, [far % 64 + n] * B)
    part = tuple(t[:, :, t0: t0 + 3].contiguous() for t in cache)
    codes, _ = ref.unpack(part)
    lo = 64 - far % 64  # the first block's old rows hold anything, and its scale with them
    for side in range(2):
        assert ref.same_codes(codes[side][:, :, 64: far % 64 + n], want.codes[side][:, :, 64: far % 64 + n]), lo
    del cache


def test_same_bits_again_and_on_another_stream(vfa):
    B, Hq, H, cap, d = 4, 8, 2, 2048, 128
    c = ref.pack(ref.random_cache(B, H, cap, d, 4))
    q, lens = rows((B, Hq, 2, d), 5).cuda(), ints([2048, 1, 900, 65])
    first = vfa.kv8_decode_fwd(q, c, lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = vfa.kv8_decode_fwd(q, c, lens)
    third = vfa.kv8_decode_fwd(q, c, lens, stream=s)
    s.synchronize()
    for x in (second, third):
        assert torch.equal(first[0], x[0]) and torch.equal(first[1], x[1])


def test_two_calls_at_once(vfa):
    """Two streams, a workspace each (the wrapper's own, and given ones), many times."""
    d, Hq, H, cap = 128, 8, 2, 4096
    jobs = []
    for i, (B, n_q, ns) in enumerate(((6, 1, 8), (3, 4, 5))):
        c = ref.pack(ref.random_cache(B, H, cap, d, 30 + i))
        q, lens = rows((B, Hq, n_q, d), 40 + i).cuda(), ints([4096 - 600 * b for b in range(B)])
        ws = torch.empty(vfa.kv8_decode_workspace_bytes(B, Hq, n_q, d, ns), dtype=torch.uint8, device="cuda")
        jobs.append((q, c, lens, ns, ws, torch.cuda.Stream(), vfa.kv8_decode_fwd(q, c, lens, n_splits=ns)))
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        for q, c, lens, ns, ws, s, want in jobs:
            with torch.cuda.stream(s):
                got.append((want, vfa.kv8_decode_fwd(q, c, lens, n_splits=ns, workspace=ws if i % 2 else None)))
    torch.cuda.synchronize()
    for want, x in got:
        assert torch.equal(want[0], x[0]) and torch.equal(want[1], x[1])


def test_refused_tensors(vfa):
    cache = vfa.kv8_cache(2, 2, 128, 64)
    x = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    q, lens = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), ints([3, 3])
    bad = [lambda: vfa.kv8_append(x.float(), x, cache, 0, 3), lambda: vfa.kv8_append(x, x.cpu(), cache, 0, 3), lambda: vfa.kv8_append(x[:1], x, cache, 0, 3),
           lambda: vfa.kv8_append(x, x, cache, lens, 3), lambda: vfa.kv8_append(x, x, cache, lens.long(), lens.long()),
           lambda: vfa.kv8_append(x, x, cache, lens.cpu(), lens.cpu()), lambda: vfa.kv8_append(x, x, cache[:3] + (cache[3][:1],), 0, 3),
           lambda: vfa.kv8_append(x, x, cache, lens[:1], lens[:1]), lambda: vfa.kv8_read(cache, 129), lambda: vfa.kv8_read(cache, -1),
           lambda: vfa.kv8_read(cache, 3, out=(x, x[:, :, :2])), lambda: vfa.kv8_read(cache, 3, seq_lens=lens.float()),
           lambda: vfa.kv8_decode_fwd(q.float(), cache, 3), lambda: vfa.kv8_decode_fwd(q[:, :, :32], cache, 3), lambda: vfa.kv8_decode_fwd(q[:1], cache, 3),
           lambda: vfa.kv8_decode_fwd(q, cache, 3, out=x), lambda: vfa.kv8_decode_fwd(q, cache, 3, lse=x), lambda: vfa.kv8_decode_fwd(q, cache, lens.cpu()),
           lambda: vfa.kv8_decode_fwd(q, cache, 3, n_splits=2, workspace=torch.empty(1 << 16, dtype=torch.uint8)),
           lambda: vfa.qk_norm_rope_fwd(x, x[:, :, :, ::2]), lambda: vfa.qk_norm_rope_fwd(x, x.cpu()), lambda: vfa.qk_norm_rope_fwd(x, x, x[:1]),
           lambda: vfa.qk_norm_rope_fwd(x, x, q_weight=q[0, 0].float()), lambda: vfa.qk_norm_rope_fwd(x, x, cos_sin=torch.zeros((4, 64), device="cuda").half()),
           lambda: vfa.qk_norm_rope_fwd(x, x, cos_sin=torch.zeros(4, device="cuda")), lambda: vfa.qk_norm_rope_fwd(x, x, first_pos=lens.float()),
           lambda: vfa.qk_norm_rope_fwd(x, x, out=(x, x, None))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    codes = [(lambda: vfa.kv8_append(x, x, cache, 0, 4), -1), (lambda: vfa.kv8_append(x, x, cache, 2, 1), -1), (lambda: vfa.kv8_append(x, x, cache, 126, 129), -1),
             (lambda: vfa.kv8_decode_fwd(q, cache, 129), -1), (lambda: vfa.kv8_decode_fwd(q, cache, 3, n_splits=0), -1),
             (lambda: vfa.kv8_decode_fwd(q, cache, 3, n_splits=2, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")), -1),
             (lambda: vfa.kv8_decode_fwd(x.repeat(1, 33, 1, 1), cache, 3), -2),
             (lambda: vfa.qk_norm_rope_fwd(x, x, eps=-1.0), -1), (lambda: vfa.qk_norm_rope_fwd(x, x, cos_sin=torch.zeros((4, 72), device="cuda")), -1),
             (lambda: vfa.qk_norm_rope_fwd(x, x, norm=False, q_weight=q[0, 0].contiguous()), -1)]
    for f, code in codes:
        with pytest.raises(vfa.VfaError) as e:
            f()
        assert e.value.code == code


# ---- together --------------------------------------------------------------------------------------------------------------------

def table(n, rot):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float().cuda()


def test_serving_loop(vfa):
    """A ragged batch of prompts (normed, rotated, prefilled in bf16, written to the cache), then steps of one and of three tokens, each against 64 bits
    over what the cache stands for; the prompts' last tokens come out of both attention paths alike."""
    B, Hq, H, d, cap = 2, 8, 2, 128, 256
    cs, w = table(cap, d), (1 + 0.1 * rows((2, d), 1)).cuda()
    kw = dict(q_weight=w[0], k_weight=w[1], cos_sin=cs)
    cache, want = vfa.kv8_cache(B, H, cap, d), ref.Cache(B, H, cap, d)
    lens = [97, 64]
    x = rows((B, 97, Hq + 2 * H, d), 2).cuda()
    Q, K, V = vfa.qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq: Hq + H], x[:, :, Hq + H:], **kw)
    O, L = vfa.vfa_attn_fwd(Q, K, V)
    vfa.kv8_append(K, V, cache, ints([0, 0]), ints(lens))
    want.append(K.cpu(), V.cpu(), [0, 0], lens)
    last = torch.stack([Q[b, :, n - 2: n] for b, n in enumerate(lens)])
    O8, L8 = vfa.kv8_decode_fwd(last, cache, ints(lens))
    ref.check(O8, L8, ref.attend(last, want.values(), lens))
    for b, n in enumerate(lens):  # (8-bit keys and values: scores off by a few hundredths, values by 2^-4 at most)
        assert (O8[b].float() - O[b, :, n - 2: n].float()).abs().mean() < 0.05 * O[b, :, n - 2: n].float().abs().mean() + 0.02
    for i, step in enumerate((1, 3, 1, 1, 3)):
        x = rows((B, step, Hq + 2 * H, d), 10 + i, 1 + i).cuda()
        Q, K, V = vfa.qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq: Hq + H], x[:, :, Hq + H:], first_pos=ints(lens), **kw)
        new = [n + step for n in lens]
        vfa.kv8_append(K, V, cache, ints(lens), ints(new))
        want.append(K.cpu(), V.cpu(), lens, new)
        O, L = vfa.kv8_decode_fwd(Q, cache, ints(new))
        same_cache(cache, want, new)
        ref.check(O, L, ref.attend(Q, want.values(), new), i)
        lens = new if step == 1 else [n + 1 for n in lens]  # (two of three drafts are refused)


def test_step_in_a_graph(vfa):
    """A whole step captured once; lengths and inputs change between the replays, with eager steps on a cache of its own beside them."""
    B, Hq, H, d, cap = 3, 8, 2, 64, 256
    cs = table(cap, d)

    def step(x, cache, lens, new, ws, out, lse):
        Q, K, V = vfa.qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq: Hq + H], x[:, :, Hq + H:], norm=False, cos_sin=cs, first_pos=lens)
        vfa.kv8_append(K, V, cache, lens, new)
        vfa.kv8_decode_fwd(Q, cache, new, n_splits=4, workspace=ws, out=out, lse=lse)

    caches = [vfa.kv8_cache(B, H, cap, d) for _ in range(2)]
    for c in caches:
        for t in c:
            t.zero_()
    lens, new = ints([0, 60, 126]), ints([1, 61, 127])
    x = rows((B, 1, Hq + 2 * H, d), 0).cuda()
    outs = [torch.empty((B, Hq, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lses = [torch.empty((B, Hq, 1), device="cuda") for _ in range(2)]
    spaces = [torch.empty(vfa.kv8_decode_workspace_bytes(B, Hq, 1, d, 4), dtype=torch.uint8, device="cuda") for _ in range(2)]
    step(x, caches[1], lens, new, spaces[1], outs[1], lses[1])  # (loads the kernels)
    for t in caches[1]:
        t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, caches[0], lens, new, spaces[0], outs[0], lses[0])
    for i in range(6):
        x.copy_(rows(x.shape, 20 + i, 1 + 5 * i).cuda())
        graph.replay()
        step(x, caches[1], lens, new, spaces[1], outs[1], lses[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]), i
        assert all(torch.equal(a, b) for a, b in zip(*caches)), i
        lens += 1
        new += 1


# ---- values at the top of bf16 ---------------------------------------------------------------------------------------------------

def top_block(c, b, t, seed):
    """Block t of sequence b gets the largest exponent that writing gives, 120, and values of some 2^120."""
    for h in range(c.codes[1].shape[1]):
        g = torch.Generator().manual_seed(seed + h)
        c.codes[1][b, h, 64 * t: 64 * t + 64] = ref.nearest(torch.randn((64, c.codes[1].shape[3]), generator=g, dtype=ref.F64))
        c.exp[1][b, h, t] = 120


@pytest.mark.parametrize("d,g,n_q", [(64, 2, 4), (128, 6, 4), (64, 5, 11), (128, 3, 30)])
@pytest.mark.parametrize("n_splits", [1, 2])
def test_top_of_bf16_in_a_draft(vfa, d, g, n_q, n_splits):
    """Codes of 256 and 448 under 2^120, which bf16 would take for infinities, in the second and third of the last four new tokens: those before them
    do not see them, and no other feature is spoiled for those who do."""
    B, H, cap = 2, 1, 192
    lens = [66, 140]
    c = ref.random_cache(B, H, cap, d, 7)
    for b, n in enumerate(lens):
        for t in sorted({(n - 3) // 64, (n - 2) // 64}):
            top_block(c, b, t, 10 * b + t)
        c.codes[1][b, :, n - 3, 5] = 0x78
        c.codes[1][b, :, n - 2, d - 1] = 0xfe
    q = rows((B, g, n_q, d), 8, 0.4).cuda()
    O, L = vfa.kv8_decode_fwd(q, ref.pack(c), ints(lens), n_splits=n_splits)
    o, l, a = ref.attend(q, c.values(), lens)
    first = n_q - 3  # (the first token that sees one)
    ref.check(O[:, :, :first], L[:, :, :first], (o[:, :, :first], l[:, :, :first], a[:, :, :first]))
    other = [f for f in range(d) if f not in (5, d - 1)]
    ref.check(O[..., other], L, (o[..., other], l, a[..., other]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,n", [(1, 200), (3, 200), (20, 200), (1, 40)])
def test_top_of_bf16_under_a_weight_of_zero(vfa, d, n_q, n):
    """A key so far below the others that its weight is zero, with a value that bf16 would take for an infinity."""
    c = ref.random_cache(1, 2, 256, d, 9)
    c.codes[0].zero_()
    c.codes[0][:, :, 10] = 0xfe  # -448
    c.exp[0].zero_()
    top_block(c, 0, 0, 3)
    c.codes[1][0, :, 10, ::3] = 0x7e
    q = torch.full((1, 4, n_q, d), 4.0, dtype=torch.bfloat16).cuda()
    for ns in (1, 2):
        O, L = vfa.kv8_decode_fwd(q, ref.pack(c), n, n_splits=ns)
        ref.check(O, L, ref.attend(q, c.values(), [n]))


# ---- numbers past the range of their type ----------------------------------------------------------------------------------------

def test_lengths_past_32_bits(vfa):
    """A length or position that does not fit into an int is refused as one that does not fit into the cache is, not taken by its low bits."""
    cache = vfa.kv8_cache(1, 2, 128, 64)
    for t in cache:
        t.zero_()
    x, q = torch.ones((1, 2, 3, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    before = [t.clone() for t in cache]
    cs = torch.zeros((4, 64), device="cuda")
    for big in (2 ** 31, 2 ** 32, 2 ** 32 + 3, 2 ** 40, -2 ** 32, -2 ** 63, 10 ** 30):
        for f in (lambda: vfa.kv8_append(x, x, cache, 0, big), lambda: vfa.kv8_append(x, x, cache, big, big + 3), lambda: vfa.kv8_decode_fwd(q, cache, big),
                  lambda: vfa.kv8_read(cache, 3, seq_lens=big), lambda: vfa.qk_norm_rope_fwd(x, x, cos_sin=cs, first_pos=big),
                  lambda: vfa.kv8_decode_fwd(q, cache, 3, n_splits=2 ** 32 + 1)):
            with pytest.raises(vfa.VfaError) as e:
                f()
            assert e.value.code == -1
    one = x[:, :, :1].expand(1, 2, 2 ** 32, 64)
    with pytest.raises(vfa.VfaError):
        vfa.kv8_append(one, one, cache, ints([0]), ints([3]))
    assert all(torch.equal(a, b) for a, b in zip(cache, before))


# ---- weights ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,n_q", [(1, 1), (4, 1), (8, 1), (1, 8), (2, 3), (7, 1)])
@pytest.mark.parametrize("n_splits", [1, 3])
def test_weights_of_up_to_eight_rows(vfa, d, g, n_q, n_splits):
    """Up to eight rows of a KV head have their weights in two halves of bf16, 2^-14 of each in all.  Scores are sums of d products in 32 bits (2^-17 of the
    terms' size, in the weight and in the sum that divides it), the rest (exponentials, sums of up to 130 keys) below 2^-16; O is rounded once."""
    lens = [1, 2, 3, 4, 5, 9, 17, 64, 65, 130]
    B, H, cap = len(lens), 2, 192
    c = ref.random_cache(B, H, cap, d, d + g)
    q = rows((B, g * H, n_q, d), n_q, 0.2).cuda()
    O, L = vfa.kv8_decode_fwd(q, ref.pack(c), ints(lens), n_splits=n_splits)
    K, V = c.values()
    o, l, a = ref.attend(q, [K, V], lens)
    terms = (q.double().cpu().abs().reshape(B, H, -1, d) @ K.abs().transpose(2, 3)).amax().item() * d ** -0.5
    off = (O.double().cpu() - o).abs() - (2.0 ** -14 + 2.0 ** -16 * (1 + terms)) * a - 2.0 ** -8 * o.abs()
    assert terms < 16 and (off <= 0).all(), (terms, off.max().item())
    ref.check(O, L, (o, l, a))
