"""Storing into 16-bit blocks, attention over them with what every block gathers, and eviction, written out plainly in 64 bits on the CPU: the definition
that the kernels are held to.  Besides a result, `attend` gives the bound that the kernels' arithmetic allows (`Bound`)."""
import math
from dataclasses import dataclass

import torch


def write(cache, new, slots):
    """A copy of cache [L][NB][T][H][128] with new [L][N][H][128] in the slots."""
    cache = cache.clone()
    L, NB, T = cache.shape[:3]
    for n, slot in enumerate(slots.tolist()):
        if 0 <= slot < NB * T:
            cache[:, slot // T, slot % T] = new[:, n]
    return cache


@dataclass
class Bound:
    """What a result may be off by, with h half a step of the output's type (relative), one rounding of the result: h |out|.

    A score is a sum of 128 products in fp32, off by at most 2^-17 of the sum of their magnitudes (128 roundings of 2^-24), and is
    taken to a power of two's exponent with roundings of 2^-24 of its size; the power itself is off by 2^-22 at most (`off`).  These are relative errors
    of a probability, and reach the output times sum p |v| (twice: once through the sum of the weights).  fp32 sums of n terms: n 2^-24, in chains
    of at most 2^11 here.  Probabilities: rounded to the 16-bit type where a call has many rows, and to the sum of two such numbers where it
    has few.  What a block gathers is a sum of probabilities, each off by 2 `off` at most, and takes part in no 16-bit rounding."""
    out: torch.Tensor
    lse: torch.Tensor
    weights: torch.Tensor


def attend(q, k, v, tables, ctx_len, starts, scale, window, many, tiny=2.0 ** -24, gathered=None):
    """out, lse [L][N][heads](..[128]) and weights [L][R][E] in 64 bits, and their Bound; rows of no request are NaN in `out`.
    tiny: what an output may be off by beside its relative bound."""
    q64, tables, k, v = q.cpu().double(), tables.cpu().long(), k.cpu(), v.cpu()
    L, N, heads, D = q64.shape
    NB, T, H = k.shape[1:4]
    R, E = tables.shape[1:]
    g, h = heads // H, torch.finfo(q.dtype).eps / 2
    out, lse = torch.full((L, N, heads, D), math.nan, dtype=torch.float64), torch.full((L, N, heads), math.nan, dtype=torch.float64)
    weights = torch.zeros((L, R, E), dtype=torch.float64) if gathered is None else gathered.cpu().double().clone()
    b_out, b_lse, b_weights = torch.zeros_like(out), torch.zeros_like(lse), weights.abs() * 2.0 ** -22
    h_p = h if many else h * h
    for l in range(L):
        for r, n in enumerate(ctx_len):
            m = starts[r + 1] - starts[r]
            n = max(n, 0)
            held = min(n, E * T)
            ids = tables[l, r, :(held + T - 1) // T]
            there = (ids >= 0) & (ids < NB)
            entry = torch.nonzero(there).flatten()
            key = (entry[:, None] * T + torch.arange(T)).flatten()
            key, in_entry = key[key < held], entry.repeat_interleave(T)[key < held]
            # (places behind the context are the last ones: cut off by their number)
            kk, vv = (x[l, ids[entry]].reshape(-1, H, D)[:key.numel()].double() for x in (k, v))
            for j in range(m):
                pos = n - m + j
                seen = key <= pos
                if window:
                    seen &= key > pos - window
                at = starts[r] + j
                if not seen.any():
                    out[l, at], lse[l, at] = 0, -math.inf
                    continue
                e = in_entry[seen]
                for kv in range(H):
                    x, a, b = q64[l, at, kv * g:(kv + 1) * g], kk[seen, kv], vv[seen, kv]
                    s = x @ a.T * scale                                                     # [g][keys]
                    p = torch.softmax(s, -1)
                    rows = slice(kv * g, (kv + 1) * g)
                    out[l, at, rows], lse[l, at, rows] = p @ b, torch.logsumexp(s, -1)
                    off = 2.0 ** -17 * (x.abs() @ a.abs().T).amax(-1) * scale + 2.0 ** -22 * (s.abs().amax(-1) * 1.45 + 32) + 2.0 ** -13
                    b_out[l, at, rows] = h * out[l, at, rows].abs() + (h_p + 2 * off)[:, None] * (p @ b.abs()) + tiny
                    b_lse[l, at, rows] = off + 2.0 ** -22 * lse[l, at, rows].abs()
                    weights[l, r].index_add_(0, e, p.sum(0))
                    b_weights[l, r].index_add_(0, e, (p * (2 * off[:, None] + 2.0 ** -20)).sum(0) + 2.0 ** -60)
    return out, lse, weights, Bound(b_out, b_lse, b_weights)


def order(w):
    """A weight's place in the order that entries leave in: NaN behind every number, -0 and 0 alike."""
    return (1, 0.0) if math.isnan(w) else (0, w + 0.0)


def evict(tables, weights, ctx_len, keep, refcount, T, n_first, n_last):
    """tables, refcount, n_evicted after an eviction, row by row."""
    tables, refcount = tables.clone(), refcount.clone()
    L, R, E = tables.shape
    NB = refcount.shape[1]
    count = torch.zeros((L, R), dtype=torch.int32)
    for l in range(L):
        for r in range(R):
            used = min(E, -(-max(0, ctx_len[r]) // T))
            row = tables[l, r].tolist()
            held = [e for e in range(used) if 0 <= row[e] < NB]
            may = [e for e in held if n_first <= e < used - n_last]
            n = min(max(0, len(held) - max(0, keep[r])), len(may))
            for e in sorted(may, key=lambda e: (order(weights[l, r, e].item()), e))[:n]:
                refcount[l, row[e]] -= 1
                tables[l, r, e] = -1
            count[l, r] = n
    return tables, refcount, count
