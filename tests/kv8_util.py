"""The 8-bit cache and the operators around it in plain 64-bit torch: a second way to everything that the kernels compute."""
import math

import torch

E_MIN = -117
F64 = torch.float64

_pos = [(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)]
_pos[127] = math.nan
E4M3 = torch.tensor(_pos + [-v for v in _pos], dtype=F64)  # value of each code


def nearest(x):
    """Code of the E4M3 value nearest to x (64 bits), the even code of two equally near ones, saturated; a NaN for a NaN."""
    v = E4M3[:127]
    a = torch.nan_to_num(x.abs(), nan=0.0, posinf=math.inf).clamp(max=448.0)
    up = torch.searchsorted(v, a.contiguous()).clamp(max=126)
    down = (up - 1).clamp(min=0)
    du, dd = v[up] - a, a - v[down]
    code = torch.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, down)
    code = torch.where(x.isnan(), 127, code)
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


class Cache:
    """The cache as codes [B, H, n_cap, d] and exponents [B, H, T], written row by row by its definition."""

    def __init__(self, B, H, n_cap, d):
        self.codes = [torch.zeros((B, H, n_cap, d), dtype=torch.uint8) for _ in range(2)]
        self.exp = [torch.zeros((B, H, n_cap // 64), dtype=torch.int32) for _ in range(2)]

    def append(self, K, V, old, new):
        for x, C, E in zip((K, V), self.codes, self.exp):
            for b, (o, n) in enumerate(zip(old, new)):
                for t in range(o // 64, -(-n // 64)) if n > o else ():
                    r0, r1 = max(o, 64 * t), min(n, 64 * t + 64)
                    rows = x[b, :, r0 - o: r1 - o].double().cpu()
                    for h in range(C.shape[1]):
                        a = torch.where(rows[h].isfinite(), rows[h].abs(), 0).max().item()
                        e = E_MIN
                        while a > 448 * 2.0 ** e:
                            e += 1
                        if r0 > 64 * t:
                            was = int(E[b, h, t])
                            if e > was:
                                C[b, h, 64 * t: r0] = nearest(E4M3[C[b, h, 64 * t: r0].long()] * 2.0 ** (was - e))
                            e = max(e, was)
                        C[b, h, r0:r1] = nearest(rows[h] * 2.0 ** -e)
                        E[b, h, t] = e

    def values(self):
        return [E4M3[c.long()] * 2.0 ** e.double().repeat_interleave(64, 2)[..., None] for c, e in zip(self.codes, self.exp)]


def place(key):
    return key % 16 // 4 * 16 + key // 16 * 4 + key % 4


def unpack(cache):
    """Codes of a cache of the library as [B, H, n_cap, d] (keys, values), and its exponents, on the host."""
    K8, V8, KS, VS = (t.cpu() for t in cache)
    B, H, T = KS.shape
    k = K8.permute(0, 1, 2, 4, 3, 5).reshape(B, H, 64 * T, -1)
    v = V8[..., place(torch.arange(64))].transpose(3, 4).reshape(B, H, 64 * T, -1)
    return [k, v], [KS.int() - 127, VS.int() - 127]


def pack(ref):
    """A library cache on the GPU with the contents of a Cache."""
    k, v = ref.codes
    B, H, n, d = k.shape
    K8 = k.reshape(B, H, n // 64, 64, d // 64, 64).transpose(3, 4).contiguous()
    V8 = torch.empty((B, H, n // 64, d, 64), dtype=torch.uint8)
    V8[..., place(torch.arange(64))] = v.reshape(B, H, n // 64, 64, d).transpose(3, 4)
    return tuple(t.cuda() for t in (K8, V8, (ref.exp[0] + 127).to(torch.uint8), (ref.exp[1] + 127).to(torch.uint8)))


def random_cache(B, H, n_cap, d, seed):
    """A Cache full of random codes (no NaN) with exponents around those of unit values."""
    g = torch.Generator().manual_seed(seed)
    ref = Cache(B, H, n_cap, d)
    for i in range(2):
        x = torch.randn((B, H, n_cap, d), generator=g, dtype=F64) * 100
        ref.codes[i] = nearest(x)
        ref.exp[i] = torch.randint(-8, -5, ref.exp[i].shape, generator=g, dtype=torch.int32)
    return ref


def same_codes(a, b):
    """Equal as values, and a NaN (of either sign) where the other is one."""
    nan_a, nan_b = a % 128 == 127, b % 128 == 127
    return torch.equal(nan_a, nan_b) and torch.equal(a[~nan_a], b[~nan_b])


def attend(q, values, lens, scale=None):
    """O, LSE [B, Hq, n_q, d] and the bound's average of |v|, in 64 bits; q is a bf16 tensor."""
    K, V = values
    B, Hq, n_q, d = q.shape
    g = Hq // K.shape[1]
    O, A = torch.zeros(q.shape, dtype=F64), torch.zeros(q.shape, dtype=F64)
    L = torch.full(q.shape[:3], -math.inf, dtype=F64)
    for b in range(B):
        for t in range(n_q):
            n = lens[b] - n_q + 1 + t
            if n <= 0:
                continue
            for h in range(Hq):
                x = K[b, h // g, :n] @ q[b, h, t].double().cpu() * (d ** -0.5 if scale is None else scale)
                L[b, h, t] = torch.logsumexp(x, 0)
                p = (x - L[b, h, t]).exp()
                O[b, h, t], A[b, h, t] = p @ V[b, h // g, :n], p @ V[b, h // g, :n].abs()
    return O, L, A


def check(O, L, ref, what=""):
    """A weight is rounded to bf16 (2^-8 of it), O once more; 2^-11 of the average of |v| for scores and sums in 32 bits (exponents up to
    some tens, 128 products of 2^-24 each)."""
    o, l, a = ref
    got, lse = O.double().cpu().reshape(o.shape), L.double().cpu().reshape(l.shape)
    nan = o.isnan()
    assert torch.equal(got.isnan(), nan), what
    assert torch.equal(lse.isneginf(), l.isneginf()) and torch.equal(lse.isnan(), l.isnan()), what
    off = (got - o).abs() - (2.0 ** -8 + 2.0 ** -11) * a - 2.0 ** -8 * o.abs()
    assert (off[~nan] <= 0).all(), (what, off[~nan].max().item())
    fin = l.isfinite()
    assert (lse[fin] - l[fin]).abs().max() <= 1e-3 if fin.any() else True, what


def norm_rope(x, w, eps, cos_sin, interleaved, first, norm=True):
    """[B, N, H, d] -> [B, H, N, d] in 64 bits, and the size of the terms that each feature is made of."""
    z = x.double().cpu()
    B, N, H, d = z.shape
    if norm:
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt()
        if w is not None:
            z = z * w.double().cpu()
    y, size = z.clone(), z.abs()
    if cos_sin is not None:
        cs = cos_sin.double().cpu()
        rot = cs.shape[1]
        for b in range(B):
            for n in range(N):
                row = cs[min(max(first[b] + n, 0), cs.shape[0] - 1)]
                for i in range(rot // 2):
                    a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
                    y[b, n, :, a] = z[b, n, :, a] * row[i] - z[b, n, :, c] * row[rot // 2 + i]
                    y[b, n, :, c] = z[b, n, :, c] * row[i] + z[b, n, :, a] * row[rot // 2 + i]
                    s = z[b, n, :, a].abs() + z[b, n, :, c].abs()
                    size[b, n, :, a], size[b, n, :, c] = s, s
    return y.transpose(1, 2), size.transpose(1, 2)
