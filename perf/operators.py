"""The serving operators around the 8-bit cache, timed through the public binding and through plain torch.

By kind (`"do"` of a case):
  rope     projected queries, keys and values of new tokens -> RMS norm of each head's queries and keys, rotation by position, and the
           head-major layout of the attention calls (`qk_norm_rope_fwd`)
  append   new rows of keys and values -> E4M3 codes in the cache, one power-of-two scale for every 64 tokens of a KV head
           (`kv8_append`); the rows before them in a block that has to take a larger scale are coded again
  read     the cache's rows as bf16 again (`kv8_read`)
  decode   attention of each sequence's newest tokens over the cache (`kv8_decode_fwd`)

The cache is (K8, V8, KS, VS): K8 [B, Hkv, T, d / 64, 64 keys, 64 features], V8 [B, Hkv, T, d features, 64 keys] with key
16 t + 4 g + r of a block at place 16 g + 4 t + r, and the scales' exponents + 127 in KS, VS [B, Hkv, T] (T blocks of 64 tokens).
"""
import math

import torch

own = False

BN = 64          # tokens of a block
E_MIN = -117     # smallest exponent of a block's scale


def listed():
    return [
        # one serving step of sixteen sequences: their new tokens on the way from the projection to the cache
        dict(name="rope_step_16", do="rope", B=16, N=1, Hq=32, Hkv=8, d=128, rot=128, pairs="half", n_pos=8192),
        # a batch of long prompts, grouped heads (the package's headline shape)
        dict(name="rope_prompt_2x16k", do="rope", B=2, N=16384, Hq=32, Hkv=8, d=128, rot=128, pairs="half", n_pos=16384),
        # a small model with 64-wide heads that rotates a part of each head, neighbouring pairs, a ragged prompt
        dict(name="rope_d64_3x777", do="rope", B=3, N=777, Hq=16, Hkv=4, d=64, rot=32, pairs="next", n_pos=4096),
        # the same step's keys and values written, each sequence at its own length
        dict(name="append_step_16", do="append", B=16, n=1, Hkv=8, d=128, cap=8192, lo=200),
        # the prompts written at once
        dict(name="append_prompt_2x16k", do="append", B=2, n=16384, Hkv=8, d=128, cap=16384, lo=0),
        # drafted tokens that run over the end of a block, one KV head per query head
        dict(name="append_draft_d64_8x5", do="append", B=8, n=5, Hkv=16, d=64, cap=4160, lo=900),
        # a prompt's cache read back in bf16, for a pass that takes bf16
        dict(name="read_2x16k", do="read", B=2, n=16384, Hkv=8, d=128, cap=16384, lo=16384),
        # a ragged batch read back
        dict(name="read_d64_3x2500", do="read", B=3, n=2500, Hkv=4, d=64, cap=2560, lo=100),
        # one user with a small context: launches and latency count
        dict(name="decode_1x2k", do="decode", B=1, Hq=32, Hkv=8, d=128, cap=4096, lo=2048, hi=2048, nq=1),
        # a small batch with long contexts, 256 MiB of cache a step
        dict(name="decode_4x32k", do="decode", B=4, Hq=32, Hkv=8, d=128, cap=32768, lo=32768, hi=32768, nq=1),
        # continuous batching: sixteen sequences, lengths from a few hundred keys to the capacity
        dict(name="decode_ragged_16", do="decode", B=16, Hq=32, Hkv=8, d=128, cap=8192, lo=200, hi=8192, nq=1),
        # four drafted tokens a sequence, 64-wide heads, a fill that is no multiple of a block
        dict(name="decode_draft_d64_8x4k", do="decode", B=8, Hq=16, Hkv=16, d=64, cap=8192, lo=4001, hi=4001, nq=4),
    ]


HEADS = [(32, 8), (32, 32), (16, 16), (16, 4), (24, 8), (64, 8), (8, 1), (12, 12)]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["rope", "append", "read", "decode", "decode"])
    Hq, Hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    if do == "rope":
        N = _spread(rng, 1, 8192)
        B = max(1, min(_spread(rng, 1, 64), (1 << 27) // (N * (Hq + 2 * Hkv) * d)))
        rot = rng.choice([d, d, d // 2, 16])
        return dict(do=do, B=B, N=N, Hq=Hq, Hkv=Hkv, d=d, rot=rot, pairs=rng.choice(["half", "next"]), n_pos=N + _spread(rng, 1, 8192))
    if do in ("append", "read"):
        n = _spread(rng, 1, 8192)
        lo = rng.choice([0, _spread(rng, 1, 4096)]) if do == "append" else _spread(rng, 1, n)
        cap = -(-(n + lo + rng.randint(0, 200)) // BN) * BN
        B = max(1, min(_spread(rng, 1, 64), (1 << 25) // (cap * Hkv * d)))
        return dict(do=do, B=B, n=n, Hkv=Hkv, d=d, cap=cap, lo=lo)
    hi = _spread(rng, 1, 32768)
    cap = -(-(hi + rng.randint(0, 500)) // BN) * BN
    B = max(1, min(_spread(rng, 1, 128), (1 << 27) // (cap * Hkv * d)))
    nq = min(32 * Hkv // Hq, rng.choice([1, 1, 1, 2, 3, 5, 8]))
    return dict(do=do, B=B, Hq=Hq, Hkv=Hkv, d=d, cap=cap, lo=rng.choice([hi, _spread(rng, 1, hi)]), hi=hi, nq=nq)


def _appended(c):
    """Old and new lengths of an append's sequences, known from the case alone."""
    lo, room = c["lo"], c["cap"] - c["n"]
    old = [lo + (37 * b) % (room - lo + 1) if lo else 0 for b in range(c["B"])]
    return old, [o + c["n"] for o in old]


def _lengths(c):
    """Lengths of a read's or a decode's sequences."""
    lo, hi = c["lo"], c.get("hi", c.get("n"))
    return [hi - (hi - lo) * b // max(1, c["B"] - 1) for b in range(c["B"])]


# ---- plain form ------------------------------------------------------------------------------------------------------------------


def _keys_out(K8):
    """[B, H, T, d / 64, 64, 64] -> [B, H, T, 64 keys, d]"""
    return K8.transpose(3, 4).reshape(*K8.shape[:3], BN, -1)


def _keys_in(x):
    return x.reshape(*x.shape[:4], -1, BN).transpose(3, 4).contiguous()


def _values_out(V8):
    """[B, H, T, d, 64 places] -> [B, H, T, 64 keys, d]"""
    B, H, T, d, _ = V8.shape
    return V8.reshape(B, H, T, d, 4, 4, 4).permute(0, 1, 2, 5, 4, 6, 3).reshape(B, H, T, BN, d)


def _values_in(x):
    B, H, T, _, d = x.shape
    return x.reshape(B, H, T, 4, 4, 4, d).permute(0, 1, 2, 6, 4, 3, 5).reshape(B, H, T, d, BN).contiguous()


def _two_to(e):
    return torch.exp2(e.float())


def _exponent(x):
    """The exponent of the scale for the finite elements of the last two axes."""
    a = torch.where(torch.isfinite(x), x.abs(), 0).amax((-2, -1)) / 448
    m, e = torch.frexp(a)              # a = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(a == 0, E_MIN, e).clamp(min=E_MIN)


def _codes(x):
    """fp32 -> E4M3, nearest even, saturated"""
    return torch.where(x.isnan(), x, x.clamp(-448, 448)).to(torch.float8_e4m3fn)


def _plain_append(s):
    K8, V8, KS, VS = s["cache"]
    old, new, n = s["old"], s["new"], s["K"].shape[2]
    B, H, T = KS.shape
    nt = (n + BN - 2) // BN + 1                                         # blocks that n rows can reach
    dev = K8.device
    bi, hi = torch.arange(B, device=dev)[:, None, None], torch.arange(H, device=dev)[None, :, None]
    tile = (old[:, None] // BN + torch.arange(nt, device=dev))          # [B, nt]
    row = tile[:, :, None] * BN + torch.arange(BN, device=dev)          # [B, nt, 64]
    fresh = ((row >= old[:, None, None]) & (row < new[:, None, None]))[:, None, :, :, None]
    before = (row < old[:, None, None])[:, None, :, :, None]
    live = (tile * BN < new[:, None])[:, None, :].expand(B, H, nt)
    at = (bi.expand(B, H, nt)[live], hi.expand(B, H, nt)[live], tile.clamp(max=T - 1)[:, None, :].expand(B, H, nt)[live])
    src = (row - old[:, None, None]).clamp(0, n - 1).reshape(B, 1, -1, 1)
    for x, C, S, out_of, into in ((s["K"], K8, KS, _keys_out, _keys_in), (s["V"], V8, VS, _values_out, _values_in)):
        d = x.shape[3]
        x = x.float().gather(2, src.expand(B, H, -1, d)).reshape(B, H, nt, BN, d)
        x = torch.where(fresh, x, 0)
        was = S[bi, hi, tile.clamp(max=T - 1)[:, None, :]].to(torch.int32) - 127
        codes = out_of(C[bi, hi, tile.clamp(max=T - 1)[:, None, :]].view(torch.float8_e4m3fn).float())
        e = _exponent(x)
        e = torch.where(before.any(3).squeeze(-1), torch.maximum(e, was), e)
        again = before & (e > was)[..., None, None]
        new_codes = _codes(x * _two_to(-e)[..., None, None])
        old_codes = _codes(codes * _two_to(was - e)[..., None, None])
        codes = torch.where(fresh, new_codes.float(), torch.where(again, old_codes.float(), codes)).to(torch.float8_e4m3fn)
        C[at] = into(codes.view(torch.uint8))[live]
        S[at] = (e + 127).to(torch.uint8)[live]
    return _cache_values(s["cache"])


def _cache_values(cache):
    K8, V8, KS, VS = cache
    return {"K": K8.view(torch.float8_e4m3fn), "V": V8.view(torch.float8_e4m3fn), "KS": KS, "VS": VS}


def _cache_floats(cache, n):
    """fp32 [B, H, n, d] of keys and values"""
    K8, V8, KS, VS = cache
    T = -(-n // BN)
    K = _keys_out(K8[:, :, :T].view(torch.float8_e4m3fn).float()) * _two_to(KS[:, :, :T].int() - 127)[..., None, None]
    V = _values_out(V8[:, :, :T].view(torch.float8_e4m3fn).float()) * _two_to(VS[:, :, :T].int() - 127)[..., None, None]
    return K.flatten(2, 3)[:, :, :n], V.flatten(2, 3)[:, :, :n]


def _plain_read(s):
    n = s["n"]
    K, V = _cache_floats(s["cache"], n)
    there = (torch.arange(n, device=K.device) < s["lens"][:, None])[:, None, :, None]
    return torch.where(there, K, 0).to(torch.bfloat16), torch.where(there, V, 0).to(torch.bfloat16)


def _plain_decode(s):
    q, lens, cap = s["q"], s["lens"], s["cap"]
    B, Hq, nq, d = q.shape
    K, V = _cache_floats(s["cache"], cap)
    H = K.shape[1]
    key = torch.arange(cap, device=q.device)
    V = torch.where((key < lens[:, None])[:, None, :, None], V, 0)
    x = q.float().reshape(B, H, -1, d) @ K.transpose(2, 3).contiguous() * d ** -0.5
    sees = (lens[:, None] - nq + 1 + torch.arange(nq, device=q.device)).clamp(min=0)       # [B, nq]
    seen = (key < sees[:, :, None]).repeat(1, Hq // H, 1)[:, None]                         # [B, 1, g nq, cap]
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0, m))
    l = p.sum(-1, keepdim=True)
    O = torch.where(l > 0, p @ V / l, 0)
    return O.to(torch.bfloat16).reshape(B, Hq, nq, d), (m + torch.log(l)).reshape(B, Hq, nq)


def _plain_rope(s):
    B, N, Hq, d = s["q"].shape
    rot = s["cos_sin"].shape[1]
    pos = (s["first"][:, None] + torch.arange(N, device=s["q"].device)).clamp(0, s["cos_sin"].shape[0] - 1)
    cos, sin = s["cos_sin"][pos][:, :, None].chunk(2, -1)               # [B, N, 1, rot / 2]
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x = x.float()
        z = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * w.float()
        if s["next"]:
            a, b = z[..., 0:rot:2], z[..., 1:rot:2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = z[..., : rot // 2], z[..., rot // 2: rot]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        out.append(torch.cat((y, z[..., rot:]), -1).to(torch.bfloat16).transpose(1, 2).contiguous())
    return out[0], out[1], s["v"].transpose(1, 2).contiguous()


# ---- inputs ----------------------------------------------------------------------------------------------------------------------


def _cuda_ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _keys(gen, shape, dtype=torch.bfloat16):
    """Keys or values: a noisy background, some features several times larger than the others."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
    return x * (1 + 3 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.05)).to(dtype)


def _cache(gen, c, rows=True):
    B, H, T, d = c["B"], c["Hkv"], c["cap"] // BN, c["d"]
    out = []
    for into in (_keys_in, _values_in):
        C = torch.empty((B, H, T, d // BN, BN, BN) if into is _keys_in else (B, H, T, d, BN), dtype=torch.uint8, device="cuda")
        S = torch.empty((B, H, T), dtype=torch.uint8, device="cuda")
        for b in range(B):
            x = _keys(gen, (1, H, T, BN, d)).float()
            e = _exponent(x)
            C[b: b + 1] = into(_codes(x * _two_to(-e)[..., None, None]).view(torch.uint8))
            S[b: b + 1] = (e + 127).to(torch.uint8)
        out.append((C, S))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    if c["do"] == "rope":
        N, Hq = c["N"], c["Hq"]
        x = torch.randn((B, N, Hq + 2 * Hkv, d), generator=gen, device="cuda", dtype=torch.bfloat16)
        angle = torch.arange(c["n_pos"], device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
        w = 1 + 0.2 * torch.randn((2, d), generator=gen, device="cuda")
        first = [(c["n_pos"] - N) * (b + 1) // B for b in range(B)]
        return dict(do="rope", q=x[:, :, :Hq], k=x[:, :, Hq: Hq + Hkv], v=x[:, :, Hq + Hkv:], qw=w[0].to(torch.bfloat16), kw=w[1].to(torch.bfloat16),
                    eps=1e-6, cos_sin=torch.cat((angle.cos(), angle.sin()), -1).float(), next=c["pairs"] == "next", first=_cuda_ints(first))
    cache = _cache(gen, c)
    if c["do"] == "append":
        old, new = _appended(c)
        K = _keys(gen, (B, Hkv, c["n"], d))
        V = _keys(gen, (B, c["n"], 2 * Hkv, d))[:, :, Hkv:].transpose(1, 2)  # (a slice of the projection's output)
        return dict(do="append", cache=cache, K=K, V=V, old=_cuda_ints(old), new=_cuda_ints(new))
    lens = _cuda_ints(_lengths(c))
    if c["do"] == "read":
        return dict(do="read", cache=cache, n=c["n"], lens=lens)
    q = torch.randn((B, c["Hq"], c["nq"], d), generator=gen, device="cuda", dtype=torch.bfloat16) * 1.5
    return dict(do="decode", cache=cache, q=q, lens=lens, cap=c["cap"])


def run(state):
    s = state
    if own:
        import paper_2604_12798_amd as vfa
        if s["do"] == "rope":
            return vfa.qk_norm_rope_fwd(s["q"], s["k"], s["v"], q_weight=s["qw"], k_weight=s["kw"], eps=s["eps"], cos_sin=s["cos_sin"],
                                        interleaved=s["next"], first_pos=s["first"])
        if s["do"] == "append":
            return _cache_values(vfa.kv8_append(s["K"], s["V"], s["cache"], s["old"], s["new"]))
        if s["do"] == "read":
            return vfa.kv8_read(s["cache"], s["n"], seq_lens=s["lens"])
        return vfa.kv8_decode_fwd(s["q"], s["cache"], s["lens"])
    return {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}[s["do"]](s)


def work(case):
    c = case
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    if c["do"] == "rope":
        heads = B * c["N"] * (c["Hq"] + 2 * Hkv)
        return {"bytes": 4 * heads * d + 4 * min(c["n_pos"], B * c["N"]) * c["rot"], "flops": 8 * B * c["N"] * (c["Hq"] + Hkv) * d}
    if c["do"] == "append":
        return {"bytes": 2 * B * Hkv * c["n"] * d * (2 + 1), "flops": 4 * B * Hkv * c["n"] * d}
    rows = sum(_lengths(c))
    if c["do"] == "read":
        return {"bytes": 2 * Hkv * d * (rows + 2 * B * c["n"]), "flops": 2 * Hkv * rows * d}
    tiles = sum(-(-n // BN) for n in _lengths(c))
    return {"bytes": 2 * Hkv * (rows * d + tiles) + 4 * B * c["Hq"] * c["nq"] * (d + 1), "flops": 4 * rows * c["Hq"] * c["nq"] * d}


# ---- the operators' definition in 64 bits ----------------------------------------------------------------------------------------


def _e4m3_values():
    """The 128 codes from 0 up: 3 bits of mantissa, exponent bias 7, 0x7f is no number."""
    v = [(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)]
    v[127] = math.nan
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _value_of(code):
    v = _e4m3_values()
    return torch.cat((v, -v))[code.int()]


def _nearest(x):
    """The value of E4M3 nearest to each finite x, of two equally near ones that with the even code."""
    v = _e4m3_values()[:127]
    a = x.abs().clamp(max=448.0)
    up = torch.searchsorted(v, a).clamp(max=126)                     # the first value >= a
    down = (up - 1).clamp(min=0)
    du, dd = v[up] - a, a - v[down]
    take = torch.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, down)
    return v[take] * torch.where(x < 0, -1.0, 1.0)


def _place(key):
    """Where a key of a block lies in V8."""
    return key % 16 // 4 * 16 + key // 16 * 4 + key % 4


def exact(case, seed):
    s = prepare(case, seed)
    c, f64 = case, torch.float64
    if c["do"] == "rope":
        N, rot, d = c["N"], c["rot"], c["d"]
        i = torch.arange(rot // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if c["pairs"] == "next" else (i, i + rot // 2)
        p = (s["first"].long()[:, None] + torch.arange(N, device="cuda")).clamp(max=c["n_pos"] - 1)
        table = s["cos_sin"].to(f64)
        out = []
        for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
            y = torch.empty((c["B"], x.shape[2], N, d), dtype=f64, device="cuda")
            for n in range(c["B"]):
                z = x[n].transpose(0, 1).to(f64)                     # [H, N, d]
                z = z / ((z * z).sum(-1, keepdim=True) / d + s["eps"]).sqrt() * w.to(f64)
                t = table[p[n]]
                turned = torch.complex(z[..., a], z[..., b]) * torch.complex(t[:, : rot // 2], t[:, rot // 2:])
                y[n] = z
                y[n][..., a], y[n][..., b] = turned.real, turned.imag
            out.append(y)
        return out[0], out[1], s["v"].to(f64).transpose(1, 2)
    K8, V8, KS, VS = s["cache"]
    place = _place(torch.arange(BN, device="cuda"))
    if c["do"] == "append":
        old, new = _appended(c)
        codes = [_value_of(K8), _value_of(V8)]
        for x, C, S in ((s["K"], codes[0], KS), (s["V"], codes[1], VS)):
            for b in range(c["B"]):
                for t in range(old[b] // BN, -(-new[b] // BN)):
                    r0, r1 = max(old[b], t * BN), min(new[b], t * BN + BN)
                    rows = x[b, :, r0 - old[b]: r1 - old[b]].to(f64)              # [H, rows, d]
                    e = torch.ceil(torch.log2(rows.abs().amax((1, 2)) / 448)).clamp(min=E_MIN)
                    k0, k1 = r0 - t * BN, r1 - t * BN
                    if C is codes[0]:
                        block = C[b, :, t].transpose(1, 2).reshape(c["Hkv"], BN, -1)
                    else:
                        block = C[b, :, t][:, :, place].transpose(1, 2).clone()
                    if k0 > 0:
                        was = S[b, :, t].to(f64) - 127
                        e = torch.maximum(e, was)
                        block[:, :k0] = _nearest(block[:, :k0] * 2.0 ** (was - e)[:, None, None])
                    block[:, k0:k1] = _nearest(rows * 2.0 ** -e[:, None, None])
                    if C is codes[0]:
                        C[b, :, t] = block.reshape(c["Hkv"], BN, -1, BN).transpose(1, 2)
                    else:
                        C[b, :, t][:, :, place] = block.transpose(1, 2)
        return {"K": codes[0], "V": codes[1], "KS": None, "VS": None}
    lens = _lengths(c)
    n = c["n"] if c["do"] == "read" else c["cap"]
    if c["do"] == "read":
        out = [torch.zeros((c["B"], c["Hkv"], n, c["d"]), dtype=f64, device="cuda") for _ in range(2)]
    else:
        out = [torch.zeros(s["q"].shape, dtype=f64, device="cuda"), torch.full(s["q"].shape[:3], -math.inf, dtype=f64, device="cuda")]
    for b, length in enumerate(lens):
        k = _value_of(K8[b]).transpose(2, 3).flatten(3) * (2.0 ** (KS[b].to(f64) - 127))[..., None, None]
        v = _value_of(V8[b])[..., place].transpose(2, 3) * (2.0 ** (VS[b].to(f64) - 127))[..., None, None]
        k, v = k.flatten(1, 2)[:, :length], v.flatten(1, 2)[:, :length]
        if c["do"] == "read":
            out[0][b, :, :length], out[1][b, :, :length] = k, v
            continue
        q = s["q"][b].to(f64).reshape(c["Hkv"], -1, c["nq"], c["d"])
        for t in range(c["nq"]):
            sees = length - c["nq"] + 1 + t
            if sees <= 0:
                continue
            x = q[:, :, t] @ k[:, :sees].transpose(1, 2).contiguous() / math.sqrt(c["d"])
            out[0][b, :, t] = (torch.softmax(x, -1) @ v[:, :sees]).reshape(c["Hq"], c["d"])
            out[1][b, :, t] = torch.logsumexp(x, -1).reshape(c["Hq"])
    return tuple(out)
