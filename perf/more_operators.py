"""Paged cache and masked, capped or biased attention, timed through the public binding and through plain torch.

By kind (`"do"` of a case):
  append   new rows of keys and values -> their places in the pages of a pool, through each sequence's table (`kvp_append`)
  decode   attention of each sequence's newest tokens over its pages (`kvp_decode_fwd`), scores capped or with a bias by distance, or plain
  ranges   documents of a packed batch, with or without prefixes -> the keys that each row sees (`row_ranges`)
  prompt   attention of whole prompts: causal, packed documents, prefixes, no mask; capped, biased or plain scores (`masked_attn_fwd`)

A pool is (K, V) [pages, Hkv, S, d]; token n of sequence b lies in page table[b, n // S], row n % S.  A row's score with a key is
s = q . k / sqrt(d), then cap * tanh(s / cap) where there is a cap, then - slope * |distance| where there are slopes.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # one serving step of sixteen sequences: each one's new token on its way into its last page, small pages
        dict(name="append_pages_step_16", do="append", B=16, n=1, Hkv=8, d=128, page=16, cap=8192, lo=200),
        # two long prompts written at once (the package's headline shape)
        dict(name="append_pages_prompt_2x16k", do="append", B=2, n=16384, Hkv=8, d=128, page=64, cap=16384, lo=0),
        # one user with a small context: launches and latency count
        dict(name="decode_pages_1x2k", do="decode", B=1, Hq=32, Hkv=8, d=128, page=16, cap=4096, lo=2048, hi=2048, nq=1, score_cap=0.0, bias=False),
        # a small batch with long contexts, 512 MiB of pages a step
        dict(name="decode_pages_4x32k", do="decode", B=4, Hq=32, Hkv=8, d=128, page=64, cap=32768, lo=32768, hi=32768, nq=1, score_cap=0.0, bias=False),
        # continuous batching with capped scores: sixteen sequences, lengths from a few hundred keys to the capacity
        dict(name="decode_pages_cap_ragged_16", do="decode", B=16, Hq=32, Hkv=8, d=128, page=16, cap=8192, lo=200, hi=8192, nq=1, score_cap=50.0, bias=False),
        # four drafted tokens a sequence, 64-wide heads, a bias by distance, a fill that is no multiple of a page
        dict(name="decode_pages_bias_draft_d64_8x4k", do="decode", B=8, Hq=16, Hkv=16, d=64, page=32, cap=8192, lo=4001, hi=4001, nq=4, score_cap=0.0, bias=True),
        # the plan of one packed row of documents
        dict(name="ranges_docs_16k", do="ranges", B=1, N=16384, docs=24, prefix=False, causal=True, pad=0, mix=1),
        # a batch of prompts with prefixes that see each other both ways, padded at their ends
        dict(name="ranges_prefix_64x2k", do="ranges", B=64, N=2048, docs=1, prefix=True, causal=True, pad=300, mix=2),
        # a short prompt with a prefix and capped scores
        dict(name="prompt_prefix_cap_777", do="prompt", B=1, N=777, Hq=32, Hkv=8, d=128, mask="docs", docs=1, prefix=True, causal=True, pad=0, mix=3,
             score_cap=30.0, bias=False),
        # a long row of packed documents, causal in each
        dict(name="prompt_docs_16k", do="prompt", B=1, N=16384, Hq=32, Hkv=8, d=128, mask="docs", docs=6, prefix=False, causal=True, pad=0, mix=4,
             score_cap=0.0, bias=False),
        # a small model with 64-wide heads and a bias by distance
        dict(name="prompt_bias_d64_4x4k", do="prompt", B=4, N=4096, Hq=16, Hkv=16, d=64, mask="causal", score_cap=0.0, bias=True),
        # a long prompt with capped scores
        dict(name="prompt_cap_8k", do="prompt", B=1, N=8192, Hq=32, Hkv=8, d=128, mask="causal", score_cap=50.0, bias=False),
    ]


HEADS = [(32, 8), (32, 32), (16, 16), (16, 4), (24, 8), (64, 8), (8, 1), (12, 12)]
PAGES = [16, 16, 32, 64, 128, 256]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["append", "decode", "decode", "ranges", "prompt", "prompt", "prompt"])
    Hq, Hkv = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])
    page = rng.choice(PAGES)
    score_cap, bias = rng.choice([(0.0, False), (0.0, True), (20.0, False), (30.0, False), (50.0, False), (50.0, True)])
    if do == "append":
        n = _spread(rng, 1, 8192)
        lo = rng.choice([0, _spread(rng, 1, 4096)])
        cap = n + lo + rng.randint(0, 200)
        B = max(1, min(_spread(rng, 1, 64), (1 << 25) // (cap * Hkv * d)))
        return dict(do=do, B=B, n=n, Hkv=Hkv, d=d, page=page, cap=cap, lo=lo)
    if do == "decode":
        hi = _spread(rng, 1, 32768)
        cap = hi + rng.randint(0, 500)
        B = max(1, min(_spread(rng, 1, 128), (1 << 27) // (cap * Hkv * d)))
        nq = rng.choice([1, 1, 1, 2, 3, 5, 8])
        return dict(do=do, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, cap=cap, lo=rng.choice([hi, _spread(rng, 1, hi)]), hi=hi, nq=nq,
                    score_cap=score_cap, bias=bias)
    if do == "ranges":
        N = _spread(rng, 1, 32768)
        return dict(do=do, B=max(1, min(_spread(rng, 1, 256), (1 << 20) // N)), N=N, docs=_spread(rng, 1, 200), prefix=rng.random() < 0.5,
                    causal=rng.random() < 0.7, pad=rng.choice([0, N // 9]), mix=rng.randrange(1000))
    N = _spread(rng, 1, 8192)
    B = max(1, min(_spread(rng, 1, 16), int(2.7e11 / (N * N * Hq * d * 2))))
    c = dict(do=do, B=B, N=N, Hq=Hq, Hkv=Hkv, d=d, mask=rng.choice(["causal", "none", "docs", "docs"]), score_cap=score_cap, bias=bias)
    if c["mask"] == "docs":
        c.update(docs=_spread(rng, 1, 30), prefix=rng.random() < 0.4, causal=rng.random() < 0.7, pad=rng.choice([0, N // 9]), mix=rng.randrange(1000))
    return c


def _documents(c, seed):
    """Offsets of each entry's documents and their prefixes' lengths.  (What a prompt costs is known from the case alone.)"""
    offsets, prefixes = [], []
    for b in range(c["B"]):
        rng = random.Random(1000 * c["mix"] + b + (1000000 * (seed + 1) if c["do"] == "ranges" else 0))
        end = c["N"] - (rng.randint(0, c["pad"]) if c["pad"] else 0)
        o = [0] + sorted(rng.randint(0, end) for _ in range(c["docs"] - 1)) + [end]
        offsets.append(o)
        prefixes.append([rng.randint(0, o[k + 1] - o[k]) for k in range(c["docs"])] if c["prefix"] else None)
    return offsets, prefixes


def _appended(c):
    """Old and new lengths of an append's sequences, known from the case alone."""
    lo, room = c["lo"], c["cap"] - c["n"]
    old = [lo + (37 * b) % (room - lo + 1) if lo else 0 for b in range(c["B"])]
    return old, [o + c["n"] for o in old]


def _lengths(c):
    """Lengths of a decode's sequences."""
    lo, hi = c["lo"], c["hi"]
    return [hi - (hi - lo) * b // max(1, c["B"] - 1) for b in range(c["B"])]


# ---- plain form ------------------------------------------------------------------------------------------------------------------


def _plain_append(s):
    K, V, (Kp, Vp), table, old, new = s["K"], s["V"], s["cache"], s["table"], s["old"], s["new"]
    n, S = K.shape[2], Kp.shape[2]
    tok = old[:, None].long() + torch.arange(n, device=K.device)
    live = tok < new[:, None]
    page = table.long().gather(1, (tok // S).clamp(max=table.shape[1] - 1))
    at = (page[live], tok[live] % S)
    for x, pool in ((K, Kp), (V, Vp)):
        pool[at[0], :, at[1]] = x.transpose(1, 2)[live]
    return Kp, Vp


def _softmax_v(x, seen, V):
    """Weights of the seen scores x [..., rows, keys] and their sum over V [..., keys, d], and the log of the weights' sum."""
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0, m))
    l = p.sum(-1, keepdim=True)
    return torch.where(l > 0, p @ V / l, 0), (m + torch.log(l)).squeeze(-1)


def _plain_decode(s):
    q, (Kp, Vp), table, lens = s["q"], s["cache"], s["table"], s["lens"]
    B, Hq, nq, d = q.shape
    H, S = Kp.shape[1], Kp.shape[2]
    n = s["longest"]
    t = table[:, : -(-n // S)].clamp(min=0).long()
    key = torch.arange(n, device=q.device)
    there = (key < lens[:, None])[:, None, :, None]
    K, V = (torch.where(there, pool[t].float().transpose(1, 2).flatten(2, 3)[:, :, :n], 0) for pool in (Kp, Vp))
    x = q.float().reshape(B, H, -1, d) @ K.transpose(2, 3).contiguous() * d ** -0.5                # [B, H, g nq, n]
    if s["score_cap"] > 0:
        x = s["score_cap"] * torch.tanh(x / s["score_cap"])
    pos = lens[:, None].long() - nq + torch.arange(nq, device=q.device)                            # [B, nq]
    if s["slopes"] is not None:
        away = (pos[:, None, :, None] - key).abs().float()                                         # [B, 1, nq, n]
        x = x - (s["slopes"][None, :, None, None] * away).reshape(B, H, -1, n)
    seen = (key <= pos[:, :, None]).repeat(1, Hq // H, 1)[:, None]
    O, lse = _softmax_v(x, seen, V)
    return O.to(torch.bfloat16).reshape(B, Hq, nq, d), lse.reshape(B, Hq, nq)


def _plain_ranges(offsets, prefix, N, causal):
    B, n = offsets.shape[0], offsets.shape[1] - 1
    i = torch.arange(N, device=offsets.device).expand(B, N)
    k = (offsets[:, None, :] <= i[:, :, None]).sum(-1) - 1                                         # the last document that begins at or before the row
    within = (k >= 0) & (k < n)
    k = k.clamp(0, n - 1)
    lo, hi = offsets.gather(1, k).long(), offsets.gather(1, k + 1).long()
    if causal:
        both = lo + (prefix.gather(1, k) if prefix is not None else 0)
        hi = torch.maximum(i + 1, torch.minimum(both, hi))
    return torch.where(within[..., None], torch.stack((lo, hi), -1), 0).int()


def _plain_prompt(s):
    Q, K, V = s["Q"], s["K"], s["V"]
    B, Hq, N, d = Q.shape
    g = Hq // K.shape[1]
    i = torch.arange(N, device=Q.device)
    if s["ranges"] is not None:
        seen = (i >= s["ranges"][:, :, :1]) & (i < s["ranges"][:, :, 1:])                           # [B, N, N]
    else:
        seen = ((i <= i[:, None]) if s["causal"] else torch.ones((N, N), dtype=torch.bool, device=Q.device)).expand(B, N, N)
    away = (i[:, None] - i).abs().float() if s["slopes"] is not None else None
    O, lse = torch.empty_like(Q), torch.empty((B, Hq, N), device=Q.device)
    step = max(1, (1 << 28) // (N * N))  # heads at a time
    for b in range(B):
        for h in range(0, Hq, step):
            hs = slice(h, min(h + step, Hq))
            kv = torch.arange(hs.start, hs.stop, device=Q.device) // g
            x = Q[b, hs].float() @ K[b, kv].float().transpose(1, 2).contiguous() * d ** -0.5
            if s["score_cap"] > 0:
                x = s["score_cap"] * torch.tanh(x / s["score_cap"])
            if away is not None:
                x = x - s["slopes"][hs, None, None] * away
            o, lse[b, hs] = _softmax_v(x, seen[b], V[b, kv].float())
            O[b, hs] = o.to(torch.bfloat16)
    return O, lse


# ---- inputs ----------------------------------------------------------------------------------------------------------------------


def _cuda_ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _keys(gen, shape):
    """Keys or values: a noisy background, some features several times larger than the others."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    return x * (1 + 3 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.05)).to(torch.bfloat16)


def _pool(gen, c):
    """A pool that has served for a while: each sequence's pages lie anywhere in it; behind a sequence's pages its table says -1."""
    S, B = c["page"], c["B"]
    M = -(-c["cap"] // S)
    ends = _appended(c)[1] if c["do"] == "append" else _lengths(c)
    need = [-(-n // S) for n in ends]
    pages = sum(need) + sum(need) // 8 + 1
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((B, M), -1, dtype=torch.int32, device="cuda")
    first = 0
    for b, n in enumerate(need):
        table[b, :n] = order[first: first + n]
        first += n
    return tuple(_keys(gen, (pages, c["Hkv"], S, c["d"])) for _ in range(2)), table


def _slopes(c):
    if not c["bias"]:
        return None
    return 2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device="cuda") / c["Hq"])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if c["do"] == "ranges" or c.get("mask") == "docs":
        offsets, prefixes = _documents(c, seed)
        offsets = _cuda_ints(offsets)
        prefixes = _cuda_ints(prefixes) if c["prefix"] else None
    if c["do"] == "ranges":
        return dict(do="ranges", offsets=offsets, prefixes=prefixes, N=c["N"], causal=c["causal"])
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    if c["do"] == "append":
        old, new = _appended(c)
        cache, table = _pool(gen, c)
        K = _keys(gen, (B, Hkv, c["n"], d))
        V = _keys(gen, (B, c["n"], 2 * Hkv, d))[:, :, Hkv:].transpose(1, 2)  # (a slice of the projection's output)
        return dict(do="append", cache=cache, table=table, K=K, V=V, old=_cuda_ints(old), new=_cuda_ints(new))
    sharp = 6.0 if c["score_cap"] else 1.5  # (scores that are capped are large ones)
    if c["do"] == "decode":
        cache, table = _pool(gen, c)
        q = torch.randn((B, c["Hq"], c["nq"], d), generator=gen, device="cuda", dtype=torch.bfloat16) * sharp
        return dict(do="decode", cache=cache, table=table, q=q, lens=_cuda_ints(_lengths(c)), longest=c["hi"], score_cap=c["score_cap"], slopes=_slopes(c))
    N = c["N"]
    Q = torch.randn((B, c["Hq"], N, d), generator=gen, device="cuda", dtype=torch.bfloat16) * sharp
    # the ranges are the plan of the batch, which all layers use
    ranges = _plain_ranges(offsets, prefixes, N, c["causal"]) if c["mask"] == "docs" else None
    return dict(do="prompt", Q=Q, K=_keys(gen, (B, Hkv, N, d)), V=_keys(gen, (B, Hkv, N, d)), ranges=ranges, causal=c["mask"] == "causal",
                score_cap=c["score_cap"], slopes=_slopes(c))


def run(state):
    s = state
    if own:
        import paper_2604_12798_amd as vfa
        if s["do"] == "append":
            return vfa.kvp_append(s["K"], s["V"], s["cache"], s["table"], s["old"], s["new"])
        if s["do"] == "decode":
            return vfa.kvp_decode_fwd(s["q"], s["cache"], s["table"], s["lens"], score_cap=s["score_cap"], slopes=s["slopes"])
        if s["do"] == "ranges":
            return vfa.row_ranges(s["offsets"], s["N"], prefix_lens=s["prefixes"], causal=s["causal"])
        return vfa.masked_attn_fwd(s["Q"], s["K"], s["V"], causal=s["causal"], ranges=s["ranges"], score_cap=s["score_cap"], slopes=s["slopes"])
    if s["do"] == "ranges":
        return _plain_ranges(s["offsets"], s["prefixes"], s["N"], s["causal"])
    return {"append": _plain_append, "decode": _plain_decode, "prompt": _plain_prompt}[s["do"]](s)


def _row_limits(c, b, seed=0):
    """The keys [lo, hi) that each row of entry b sees."""
    N = c["N"]
    if c.get("mask", "docs") != "docs":
        return [(0, i + 1 if c["mask"] == "causal" else N) for i in range(N)]
    offsets, prefixes = _documents(c, seed)
    o, limits = offsets[b], [(0, 0)] * N
    for k in range(c["docs"]):
        for i in range(o[k], o[k + 1]):
            reach = o[k] + (prefixes[b][k] if c["prefix"] else 0)
            limits[i] = (o[k], max(i + 1, min(reach, o[k + 1])) if c["causal"] else o[k + 1])
    return limits


def work(case):
    c = case
    B = c["B"]
    if c["do"] == "ranges":
        return {"bytes": 8 * B * c["N"] + 4 * B * (c["docs"] * (2 if c["prefix"] else 1) + 1), "flops": 0}
    Hkv, d = c["Hkv"], c["d"]
    if c["do"] == "append":
        return {"bytes": 8 * B * Hkv * c["n"] * d, "flops": 0}
    if c["do"] == "decode":
        L = _lengths(c)
        return {"bytes": 4 * Hkv * sum(L) * d + 4 * sum(-(-n // c["page"]) for n in L) + 4 * B * c["Hq"] * c["nq"] * (d + 1),
                "flops": 4 * sum(L) * c["Hq"] * c["nq"] * d}
    pairs = sum(hi - lo for b in range(B) for lo, hi in _row_limits(c, b))
    return {"bytes": 4 * B * c["N"] * (c["Hq"] + Hkv) * d + 4 * B * c["Hq"] * c["N"] + (8 * B * c["N"] if c["mask"] == "docs" else 0),
            "flops": 4 * pairs * c["Hq"] * d}


# ---- the operators' definition in 64 bits ----------------------------------------------------------------------------------------


def _attend(q, k, v, lo, hi, pos, cap, slope):
    """Rows q [n, d] at positions pos over keys k, v [m, d]; each sees the keys lo <= j < hi."""
    x = q @ k.T.contiguous() / math.sqrt(q.shape[1])
    if cap > 0:
        x = cap * torch.tanh(x / cap)
    j = torch.arange(k.shape[0], device=q.device)
    if slope is not None:
        x = x - slope * (pos[:, None] - j).abs().to(torch.float64)
    x = x.masked_fill((j < lo[:, None]) | (j >= hi[:, None]), -math.inf)
    lse = torch.logsumexp(x, -1)
    return torch.exp(x - torch.where(lse == -math.inf, 0, lse)[:, None]) @ v, lse


def exact(case, seed):
    c, f64 = case, torch.float64
    if c["do"] == "ranges":
        return _cuda_ints([_row_limits(c, b, seed) for b in range(c["B"])])
    s = prepare(case, seed)
    slopes = None if c["do"] == "append" or s["slopes"] is None else s["slopes"].to(f64)
    if c["do"] == "append":
        S = c["page"]
        out = [pool.to(f64) for pool in s["cache"]]
        old, new = _appended(c)
        table = s["table"].tolist()
        for b in range(c["B"]):
            for t in range(old[b] // S, -(-new[b] // S)):
                r0, r1 = max(old[b], t * S), min(new[b], t * S + S)
                for x, pool in ((s["K"], out[0]), (s["V"], out[1])):
                    pool[table[b][t], :, r0 - t * S: r1 - t * S] = x[b, :, r0 - old[b]: r1 - old[b]].to(f64)
        return tuple(out)
    g = c["Hq"] // c["Hkv"]
    if c["do"] == "decode":
        O = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
        lse = torch.full(s["q"].shape[:3], -math.inf, dtype=f64, device="cuda")
        for b, n in enumerate(_lengths(c)):
            pages = s["table"][b, : -(-n // c["page"])].long()
            pos = torch.arange(n - c["nq"], n, device="cuda")
            for h in range(c["Hkv"]):
                k, v = (pool[pages, h].reshape(-1, c["d"])[:n].to(f64) for pool in s["cache"])
                for hq in range(h * g, h * g + g):
                    O[b, hq], lse[b, hq] = _attend(s["q"][b, hq].to(f64), k, v, torch.zeros_like(pos), pos + 1, pos, c["score_cap"],
                                                   None if slopes is None else slopes[hq])
        return O, lse
    O = torch.zeros(s["Q"].shape, dtype=f64, device="cuda")
    lse = torch.empty(s["Q"].shape[:3], dtype=f64, device="cuda")
    for b in range(c["B"]):
        limits = torch.tensor(_row_limits(c, b), device="cuda")
        for h in range(c["Hq"]):
            k, v = s["K"][b, h // g].to(f64), s["V"][b, h // g].to(f64)
            for r in range(0, c["N"], 4096):
                rows = slice(r, min(r + 4096, c["N"]))
                O[b, h, rows], lse[b, h, rows] = _attend(s["Q"][b, h, rows].to(f64), k, v, limits[rows, 0], limits[rows, 1],
                                                         torch.arange(rows.start, rows.stop, device="cuda"), c["score_cap"],
                                                         None if slopes is None else slopes[h])
    return O, lse
