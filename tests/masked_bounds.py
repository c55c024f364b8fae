"""How far masked, capped or biased attention may be off, key by key: a key's own error counts as much as its weight does, so that a far key of weight zero allows
nothing.  On the tensors' own device, in 64 bits."""
import math

import torch

from masked_util import F64, HALF_BF16, HALF_F32


def attend_by_key(q, k, v, seen, away, cap, slope, scale=None, weights=HALF_BF16):
    """As masked_util.attend: rows q [n, d] over k, v [m, d], seen [n, m], away [n, m] -> (O, LSE, tolerance of O, tolerance of LSE).

    Key j's exponent is off by up to e_j:
      its product with the row, d terms, each rounded and summed in some order, and the scale: r_j = (d + 2) half steps of the sum of the terms' magnitudes;
      a cap, which is monotone, makes of that what it makes of the ends s - r_j and s + r_j, and adds 2^-21 of itself (see masked_util);
      a bias: half steps of slope * (4 distance + 7 * 32) (see masked_util);
      the factor log2(e), the step's offset, the reference (the max, up to 8 above it) and the difference to it: four roundings of |x_j| + |max| + 8.
    The weights are w_j exp(delta_j) over their sum, |delta_j| <= e_j: the largest is w_j exp(e_j) / (w_j exp(e_j) + sum of the others' w exp(-e)), the smallest the other way round.
    LSE is off by up to log(sum w exp(e)) upwards and -log(sum w exp(-e)) downwards.  Both sums have up to m terms: 2 m roundings.  A weight is rounded for the product with V (`weights`,
    once more at 2^-8 of that, which is 1 %), and the output once."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    dev, n, m = q.device, q.shape[0], k.shape[0]
    scale = q.shape[1] ** -0.5 if scale is None else scale
    if m == 0:
        return torch.zeros((n, v.shape[1]), dtype=F64, device=dev), torch.full((n,), -math.inf, dtype=F64, device=dev), 0.0, 0.0
    x = torch.nan_to_num(q @ k.T * scale, nan=0.0, posinf=0.0, neginf=0.0)   # (what is not finite is seen by no row that is compared)
    size = (q.abs() @ torch.nan_to_num(k, nan=0.0, posinf=0.0, neginf=0.0).abs().T) * scale
    r = (q.shape[1] + 2) * HALF_F32 * torch.nan_to_num(size, nan=0.0, posinf=0.0, neginf=0.0)
    if cap:
        t = cap * torch.tanh(x / cap)
        r = torch.maximum(cap * torch.tanh((x + r) / cap) - t, t - cap * torch.tanh((x - r) / cap)) + 2.0 ** -21 * cap
        x = t
    if slope is not None:
        x = x - slope * away
        r = r + HALF_F32 * abs(slope) * (4 * away + 7 * 32)
    top = torch.where(seen, x, -math.inf).amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    e = torch.where(seen, r + 4 * HALF_F32 * (x.abs() + top.abs() + 8), 0)
    assert e.max() < 300, "exponents that fp32 does not hold"
    p = torch.where(seen, torch.exp(torch.where(seen, x - top, 0)), 0)
    l = p.sum(-1, keepdim=True)
    some = l > 0
    w = torch.where(some, p / torch.where(some, l, 1), 0)
    up, down = w * e.exp(), w * (-e).exp()
    sum_up, sum_down = up.sum(-1, keepdim=True), down.sum(-1, keepdim=True)
    most = up / (up + (sum_down - down).clamp(min=0)).clamp(min=1e-300)
    least = down / (down + (sum_up - up).clamp(min=0)).clamp(min=1e-300)
    change = torch.maximum(most - w, w - least)
    special = ~torch.isfinite(v)
    clean = torch.where(special, 0, v)
    O = w @ clean
    for j in special.any(1).nonzero().flatten().tolist():  # (0 times an infinity of a key that the row does not see is nothing)
        O = O + torch.where(seen[:, j, None] & special[j][None], v[j][None], 0)
    lse = torch.where(some, top + torch.log(torch.where(some, l, 1)), -math.inf).squeeze(-1)
    tol_o = HALF_BF16 * 1.01 * torch.nan_to_num(O, nan=0.0, posinf=0.0, neginf=0.0).abs() + ((1.01 * weights + 2.02 * m * HALF_F32) * w + change) @ clean.abs() + 1e-30
    off = torch.maximum(torch.log(torch.where(some, sum_up, 1)), -torch.log(torch.where(some, sum_down, 1))).squeeze(-1)
    tol_l = 1.01 * (off + (2 * m + 4) * HALF_F32 + 4 * HALF_F32 * torch.where(lse == -math.inf, 0, lse).abs())
    return O, lse, tol_o, tol_l


def zero_would_fail(want, lse, tol):
    """An output of 0 would not get past the tolerance, in all rows that see a key but one in a hundred.  (At the ends of scales and slopes two keys may lie so close that either may have all
    of the weight: the middle row of 97 has two farthest keys, at 48 each, and half steps of 2^18 * (4 * 48 + 7 * 32) are 6.5 nats.  Such a row is held to that.)"""
    loose = ~(torch.nan_to_num(want, nan=math.inf).abs() > tol).any(-1) & (lse != -math.inf)
    return loose.sum() <= max(1, len(lse) // 100)
