"""Attention whose outputs nearly cancel, so that a bound on them is one on the probabilities: values of magnitudes that the cache holds exactly,
with signs that bring the weighted sum of a dim close to 0 for one of the rows.  Scores are exact products (one dim of K and q).

What an output may be off by where a probability is the sum of two numbers of the 16-bit type, relative to sum p |v| (p the softmax):
  p as two numbers        (step of the type)^2: eps^2 where both are cut, as fp16's are; (eps / 2)^2 rounded, as bf16's
  p itself                the exponent is below 16 in magnitude, off by half its step, 2^-21, times log 2; the scale in it by 2^-24 of itself (exponents differ by
                          12 at most: 2^-20); a power of two by 2^-23; those that join waves likewise: 2^-19 in all, and as much again through the sum
  sums                    products are exact in fp32; 32 tokens as two numbers are 64 terms, and up to 128 tokens are one such run for each of
                          four waves: 68 roundings (which may be cuts) of 2^-23
An output itself is rounded by eps / 2 of it."""
import torch

ROUNDINGS = 68 * 2.0 ** -23 + 2 * 2.0 ** -19
TOKENS = 128


def weights(q, k):
    """Softmax [rows][n] of exact products of q [rows] and k [n], in 64 bits."""
    return torch.softmax(q.double()[:, None] * k.double()[None], 1)


def problem(rows, n, dtype, g):
    """q [rows], k [n] (one dim), v [n][128]; dim d cancels for row d % rows."""
    assert n <= TOKENS
    q = (0.3 + torch.rand(rows, generator=g)).to(dtype)
    k = torch.tensor([-3.0, -2.0, -1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0])[torch.randint(0, 11, (n,), generator=g)]
    size = torch.tensor([0.5, 1, 1.5, 2, 3, 4, 6])[torch.randint(0, 7, (n, 128), generator=g)]
    size[:, ::32] = 6                                # every group of 32 dims has the same power
    p = weights(q, k)[torch.arange(128) % rows].T    # [n][128]
    share, order = (p * size).sort(0, descending=True)
    sign, total = torch.empty(n, 128), torch.zeros(128, dtype=torch.float64)
    for i in range(n):
        s = torch.where(total > 0, -1.0, 1.0)
        total += s * share[i]
        sign.scatter_(0, order[i:i + 1], s.float()[None])
    return q, k.to(dtype), (size * sign).to(dtype)


def bound(p, v, dtype):
    """Of outputs [rows][128], with p [rows][n] and v [n][128] in 64 bits."""
    eps = torch.finfo(dtype).eps
    two = eps ** 2 if dtype == torch.float16 else (eps / 2) ** 2
    return eps / 2 * (p @ v).abs() + (two + ROUNDINGS) * (p @ v.abs()) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
