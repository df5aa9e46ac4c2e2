"""Attention whose exact results are far below the magnitudes that they are summed
from, so that the bits of the softmax weights show behind the output's rounding."""
import torch

import ref_lm as ref


def cancelling(seed, seqs, n, heads, dim, dtype):
    """(q, k, v, offsets, weights, places) of `seqs` sequences of n tokens.  All queries are the first unit vector and
    scores, at a scale of one, the first column of k: 0, a and b in [-1, 0] at three places, -300 at the others, whose
    weights are zero in fp32.  The values at the three places cancel as far as the type lets them, column by column:
    the second takes the first one away and the third what that leaves.  `weights` are the three, before their division
    by their sum, in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(seqs, n, heads, dim, generator=g)
    v = torch.randn(seqs, n, heads, dim, generator=g).to(dtype).double()
    s = -torch.rand(3, seqs, heads, generator=g).to(torch.bfloat16)
    s[0] = 0
    w = torch.exp(s.double())
    places = torch.stack([torch.randperm(n, generator=g)[:3] for _ in range(seqs)])
    k[..., 0] = -300
    at = torch.arange(seqs)
    rest = (1 + torch.rand(seqs, heads, dim, generator=g)).to(dtype).double()
    v[at, places[:, 0]] = rest
    for i in range(3):
        k[at, places[:, i], :, 0] = s[i].float()
        if i:
            x = (-rest / w[i][..., None]).to(dtype).double()
            v[at, places[:, i]] = x
            rest = rest + w[i][..., None] * x
    q = torch.zeros(seqs * n, heads, dim)
    q[..., 0] = 1
    k, v = k.flatten(0, 1).to(dtype), v.flatten(0, 1).to(dtype)
    return q.to(dtype), k, v, [n * i for i in range(seqs + 1)], w, places


def result(v, w, places, n):
    """(y, magnitudes), [sequences][heads][dim], from the three weights of each sequence and head."""
    seqs = places.shape[0]
    x = ref.f64(v).view(seqs, n, *v.shape[1:])
    picked = torch.stack([x[torch.arange(seqs), places[:, i]] for i in range(3)])
    w = (w / w.sum(0))[..., None]
    return (w * picked).sum(0), (w * picked.abs()).sum(0)


def bound(y, mag, dtype):
    """In units of 2^-24 of the magnitudes: log2 e as a constant (1.44), the score's place under the maximum (1, as it is
    under 2) and so 1.7 in the weight, the exponential (2); nine sums of three parts of three products, each cut off
    rather than rounded (18).  Zeros add nothing, the largest score is zero, and sum and quotient are errors of the
    small result itself.  With them and the output's rounding: 22, and half a step of the type."""
    return ref.half_ulp(dtype) * y.abs() + 22 * 2.0 ** -24 * mag


def cut(t, bits):
    """fp32 values rounded to so many bits."""
    m, e = torch.frexp(t.double())
    return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits).float()


def plain_f32(q, k, v, causal, window, scale, weights=lambda w: w):
    """One sequence in fp32 steps throughout, each product and each addition rounded: scores summed over the columns one
    by one, results over the keys."""
    n, hq, dim = q.shape
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    seen = (j <= i) if causal else torch.ones(n, n, dtype=torch.bool)
    if window:
        seen = seen & (j > i - window)
    y = torch.zeros(n, hq, v.shape[2])
    for h in range(hq):
        a = h // (hq // k.shape[1])
        s = torch.zeros(n, n)
        for d in range(dim):
            s += q[:, h, d, None] * k[None, :, a, d]
        s = torch.where(seen, s * scale, -float("inf"))
        w = weights(torch.exp(s - s.max(1, keepdim=True).values))
        for r in range(n):
            y[:, h] += w[:, r, None] * v[r, a]
        y[:, h] /= w.sum(1, keepdim=True)
    return y


def far(y, want):
    """Root of the mean squared error, for each head."""
    return (ref.f64(y) - want).pow(2).mean((0, 2)).sqrt()


# fp32 calls round as plain_f32() does, but for fused products (half its roundings) and the exponent in powers of two
# (one more): twice its error is a bound.
F32_CASES = [(513, 64, True, 0), (450, 128, True, 0), (300, 200, False, 0), (700, 80, True, 257), (100, 128, True, 0)]


def f32_case(n, dim):
    g = torch.Generator().manual_seed(n + dim)
    sharp = 1 + 2 * torch.rand(4, 1, generator=g)
    return (torch.randn(n, 4, dim, generator=g) * sharp, torch.randn(n, 2, dim, generator=g),
            torch.randn(n, 2, dim, generator=g))
