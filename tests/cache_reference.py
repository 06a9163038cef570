"""The 4-bit cache and the attention over it, written out plainly in 64 bits on the CPU: the definition that the kernels are held to.

Codes are found by trying all sixteen, a group's power by trying exponents from the smallest, bytes by their addresses, attention row
by row.  Besides a result, `attend` gives the bound that the kernels' arithmetic allows (`Bound`)."""
import math
from dataclasses import dataclass

import torch

RECORD = 2176
MAGNITUDES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
LIMITS = {torch.float16: (-23, 13), torch.bfloat16: (-125, 125)}


def group_power(big, dtype):
    """Exponent x of a group whose largest magnitude is `big` (a Python float); None where it is not finite."""
    if not math.isfinite(big):
        return None
    low, high = LIMITS[dtype]
    x = low
    while x < high and big > 7.0 * 2.0 ** x:
        x += 1
    return x


def quantise(x, dtype):
    """Codes [..][128] (0 to 15) and exponent bytes [..][4] of heads [..][128]."""
    g = x.double().reshape(-1, 32)
    big = g.abs().amax(1)
    powers = [group_power(v, dtype) for v in big.tolist()]
    ok = torch.tensor([p is not None for p in powers])
    p = torch.tensor([0 if p is None else p for p in powers], dtype=torch.float64)
    r = torch.where(ok[:, None], g.abs(), torch.zeros_like(g)) / torch.exp2(p)[:, None]
    distance = (r[..., None] - MAGNITUDES).abs()
    best = distance.amin(-1, keepdim=True)
    near = distance == best
    # of two equally near codes the even one
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = torch.where(ok[:, None], code + 8 * torch.signbit(g).long(), torch.zeros_like(code))
    bytes_ = torch.where(ok, p.long() + 127, torch.full_like(p.long(), 255))
    return code.reshape(x.shape).to(torch.uint8), bytes_.reshape(*x.shape[:-1], 4).to(torch.uint8)


def addresses(t):
    """For the place t of a record's 16: addresses of the bytes of K's and V's codes by dim, and of their exponents by group."""
    d, g = torch.arange(128), torch.arange(4)
    return ((d // 32 * 16 + t) * 16 + d % 32 // 2, 1024 + ((t // 4 * 16 + d // 8) * 4 + t % 4) * 4 + d % 8 // 2,
            2048 + g * 16 + t, 2112 + (t // 4 * 4 + g) * 4 + t % 4)


def write(cache, k, v, slots):
    """A copy of cache [L][NB][H][T/16][2176] (CPU) with k, v [L][N][H][128] in the slots."""
    cache = cache.clone()
    L, NB, H, tiles, _ = cache.shape
    (kc, kb), (vc, vb) = quantise(k, k.dtype), quantise(v, v.dtype)
    for n, slot in enumerate(slots.tolist()):
        if not 0 <= slot < NB * tiles * 16:
            continue
        b, tile, t = slot // (tiles * 16), slot // 16 % tiles, slot % 16
        ak, av, ek, ev = addresses(t)
        rec = cache[:, b, :, tile]
        for code, at in ((kc, ak), (vc, av)):
            rec[:, :, at[0::2]] = code[:, n, :, 0::2] | code[:, n, :, 1::2] << 4
        rec[:, :, ek] = kb[:, n]
        rec[:, :, ev] = vb[:, n]
    return cache


def read(cache, ids):
    """K and V [L][n][T][H][128] in 64 bits; blocks outside the cache are zeros."""
    cache, ids = cache.cpu(), ids.cpu()
    L, NB, H, tiles, _ = cache.shape
    there = (ids >= 0) & (ids < NB)
    rec = cache[:, torch.where(there, ids, 0).long()] if NB else torch.zeros((L, ids.numel(), H, tiles, RECORD), dtype=torch.uint8)
    out = [torch.zeros((L, ids.numel(), tiles * 16, H, 128), dtype=torch.float64) for _ in range(2)]
    d = torch.arange(128)
    for tile in range(tiles):
        for t in range(16):
            ak, av, ek, ev = addresses(t)
            for o, at, e in ((out[0], ak, ek), (out[1], av, ev)):
                code = (rec[:, :, :, tile, at].long() >> (d % 2 * 4)) & 15
                byte = rec[:, :, :, tile, e].double().repeat_interleave(32, -1)
                value = MAGNITUDES[code % 8] * torch.where(code >= 8, -1.0, 1.0) * torch.exp2(byte - 127)
                o[:, :, tile * 16 + t] = torch.where(byte == 255, math.nan, value)
    for o in out:
        o[:, ~there] = 0
    return out


@dataclass
class Bound:
    """What a result may be off by, with h half a step of the output's type (relative), one rounding of the result: h |out|.

    A score is a sum of 128 products in fp32, off by at most 2^-17 of the sum of their magnitudes (128 roundings of 2^-24), and is
    taken to a power of two's exponent with roundings of 2^-24 of its size; the power itself is off by 2^-22 at most.  Both are relative errors of a
    probability, and reach the output times sum p |v| (twice: once through the sum of the weights).  fp32 sums of n terms: n 2^-24, in chains
    of at most 2^11 here.  Probabilities: rounded to the 16-bit type where a call has many rows, and to the sum of two such numbers where it
    has few."""
    out: torch.Tensor
    lse: torch.Tensor


def attend(q, cache, tables, ctx_len, starts, scale, window, many, tiny=2.0 ** -24):
    """out, lse [L][N][heads](..[128]) in 64 bits, and their Bound; rows of no request are NaN in `out`.
    tiny: what an output may be off by beside its relative bound."""
    q64, tables = q.cpu().double(), tables.cpu()
    L, N, heads, D = q64.shape
    NB, H, T = cache.shape[1], cache.shape[2], cache.shape[3] * 16
    E, g, h = tables.shape[2], heads // H, torch.finfo(q.dtype).eps / 2
    out, lse = torch.full((L, N, heads, D), math.nan, dtype=torch.float64), torch.full((L, N, heads), math.nan, dtype=torch.float64)
    b_out, b_lse = torch.zeros_like(out), torch.zeros_like(lse)
    h_p = h if many else h * h
    cpu = cache.cpu()
    for l in range(L):
        for r, n in enumerate(ctx_len):
            m = starts[r + 1] - starts[r]
            n = max(n, 0)
            held = min(n, E * T)
            ids = tables[l, r, :(held + T - 1) // T]
            there = ((ids >= 0) & (ids < NB)).repeat_interleave(T)[:held]
            k, v = (x[0].reshape(-1, H, D)[:held] for x in read(cpu[l:l + 1], ids))
            key = torch.arange(held)
            for j in range(m):
                pos = n - m + j
                seen = there & (key <= pos)
                if window:
                    seen &= key > pos - window
                at = starts[r] + j
                for head in range(heads):
                    x, kk, vv = q64[l, at, head], k[seen, head // g], v[seen, head // g]
                    if kk.shape[0] == 0:
                        out[l, at, head], lse[l, at, head] = 0, -math.inf
                        continue
                    s = kk @ x * scale
                    p = torch.softmax(s, 0)
                    out[l, at, head], lse[l, at, head] = p @ vv, torch.logsumexp(s, 0)
                    off = (2.0 ** -17 * (kk.abs() @ x.abs()).max() * scale + 2.0 ** -22 * (s.abs().max() * 1.45 + 32) + 2.0 ** -13).item()
                    b_out[l, at, head] = h * out[l, at, head].abs() + (h_p + 2 * off) * (p @ vv.abs()) + tiny
                    b_lse[l, at, head] = off + 2.0 ** -22 * lse[l, at, head].abs()
    return out, lse, Bound(b_out, b_lse)
