"""The paged cache and masked, capped or biased attention in plain 64-bit torch, and how far a kernel may be off."""
import math

import torch

F64 = torch.float64
HALF_BF16 = 2.0 ** -8    # half a step of bf16, relative
HALF_F32 = 2.0 ** -24


def attend(q, k, v, seen, away, cap, slope, scale=None, weights=HALF_BF16):
    """Rows q [n, d] (bf16 or wider) over k, v [m, d]; seen [n, m]; away [n, m] distances.  Returns (O, LSE, tolerance of O, tolerance of LSE).

    What a kernel that holds scores and sums in 32 bits may be off by.  A score is a product of d terms, each rounded, and summed in some order: d roundings
    of at most the sum of its terms' magnitudes; one more for the scale.  A cap computes tanh(y) = 1 - 2 / (1 + e^(2 y)) times itself: an exponential, a
    sum, a reciprocal of 1 ulp and a multiply-add, 2^-21 of the cap is above their sum; an error of the score goes through it at most once.  A bias by the distance rounds the
    slope times log2(e), the distance, their product and the sum: four roundings of slope * distance.  A kernel may take it in two parts, slope times the key's place in a block
    of 32 keys, in units of raw scores, and slope times the rest, which then are up to slope * 31 and slope * (distance + 31).  The first rounds the slope over the scale, the slope in
    pieces and three products' sums (5 * 31), the rest its product and its difference to the max (2 * 31 beside the distance's own): slope * (4 * distance + 7 * 32) at most.
    The exponent's own product with log2(e) and the difference to the max round
    at the scores' magnitude, four more.  An error of e of all exponents changes a weight by e and the sum that divides by at most e: 2 e (1 % is far above the
    second order).  The row's sums have at most m terms: 2 m roundings.  `weights`: the rounding of weights for the product with V (twice where
    the max moves between them and the product, but then they are 2^-8 of the new max at most, and 2^-16 is less than 1 % of 2^-8).  Then one rounding of the output."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    scale = q.shape[1] ** -0.5 if scale is None else scale
    x = q @ k.T * scale
    nan_free = torch.nan_to_num(k, nan=0.0, posinf=0.0, neginf=0.0)
    size = (q.abs() @ nan_free.abs().T) * scale
    err = (q.shape[1] + 2) * HALF_F32 * size
    if cap:
        x = cap * torch.tanh(x / cap)
        err = err + 2.0 ** -21 * cap
    if slope is not None:
        x = x - slope * away
        err = err + HALF_F32 * abs(slope) * (4 * away + 7 * 32)
    err = err + 4 * HALF_F32 * torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0).abs()
    err = torch.where(seen, err, 0).amax(-1, keepdim=True) if k.shape[0] else torch.zeros((q.shape[0], 1), dtype=F64)
    x = torch.where(seen, x, -math.inf)
    if k.shape[0] == 0:
        return torch.zeros((q.shape[0], v.shape[1]), dtype=F64), torch.full((q.shape[0],), -math.inf, dtype=F64), 0.0, 0.0
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    w = torch.where(l > 0, p / l, torch.zeros_like(p))
    w = torch.where(seen, w, 0)
    O = torch.empty((q.shape[0], v.shape[1]), dtype=F64)
    special = ~torch.isfinite(v)
    if special.any():  # (0 times an infinity of a key that the row does not see is nothing)
        O = w @ torch.where(special, 0, v)
        for j in special.any(1).nonzero().flatten().tolist():
            O = O + torch.where(seen[:, j, None] & special[j][None], v[j][None], 0)
    else:
        O = w @ v
    lse = (m + torch.log(l)).squeeze(-1)
    spread = w @ torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0).abs()
    tol_o = HALF_BF16 * 1.01 * O.abs() + (weights + 2.02 * err + 2 * k.shape[0] * HALF_F32) * 1.01 * spread + 1e-30
    tol_l = (err.squeeze(-1) + 2 * k.shape[0] * HALF_F32 + 4 * HALF_F32 * torch.nan_to_num(lse, nan=0.0, neginf=0.0).abs() + 4 * HALF_F32) * 1.01
    return O, lse, tol_o, tol_l


def compare(got, lse, want, want_lse, tol_o, tol_l, what):
    got, lse = got.detach().cpu().to(F64), lse.detach().cpu().to(F64)
    plain = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.where(plain | want.isnan(), 0.0, got), torch.where(plain | want.isnan(), 0.0, want)), what
    off = torch.where(plain, (got - want).abs() - tol_o, -1.0)
    assert off.max() <= 0, (what, "O", off.max().item(), (off > 0).sum().item(), (off > 0).nonzero()[:4].tolist())
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty), (what, "rows that see nothing")
    assert (got[empty] == 0).all(), what
    off = torch.where(empty | ~torch.isfinite(want_lse), -1.0, (lse - want_lse).abs() - tol_l)
    assert off.max() <= 0, (what, "LSE", off.max().item())


def paged(gen, lens, Hkv, d, page, cap, holes=(), spare=3, fill=math.nan):
    """Keys and values of sequences, as lists of [Hkv, n, d], and a pool and table that hold them: pages in any order, everything else of the pool is `fill`.
    holes: (sequence, page) pairs whose entry is no page; the tokens there come back as None in `there`."""
    B, M = len(lens), -(-cap // page)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=gen).tolist()
    pool = [torch.full((n_pages, Hkv, page, d), fill, dtype=torch.bfloat16) for _ in range(2)]
    table = torch.randint(-3, 0, (B, M), generator=gen, dtype=torch.int32)
    table[:, 1::2] = n_pages + 5
    rows, there = [], []
    for b, n in enumerate(lens):
        kv = [torch.randn((Hkv, n, d), generator=gen).to(torch.bfloat16) for _ in range(2)]
        ok = torch.ones(n, dtype=torch.bool)
        for t in range(need[b]):
            at, end = t * page, min(n, t * page + page)
            if (b, t) in holes:
                ok[at:end] = False
                continue
            i = order.pop()
            table[b, t] = i
            for x, p in zip(kv, pool):
                p[i, :, : end - at] = x[:, at:end]
        rows.append(kv)
        there.append(ok)
    return rows, there, pool, table
