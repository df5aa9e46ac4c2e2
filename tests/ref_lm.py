"""Plain 64-bit CPU forms of the decoder operators, written from their
definitions in include/convsel_lm.h, with the sums that bound a kernel's error."""
import math

import numpy as np
import torch

QMAX = {"int8": 127.0, "fp8": 448.0}


def f64(t):
    return t.detach().double().cpu()


# What one rounding to the type costs at most, relative: 2^-p for p significant
# bits (8 for bf16, its leading one included; 24 for fp32).
def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def linear(x, w, b=None, activation="none", residual=None):
    """(y, bound): bound holds the magnitudes whose fp32 rounding the sum may show."""
    x, w = f64(x), f64(w)
    z, mag = x @ w.T, x.abs() @ w.T.abs()
    if b is not None:
        z, mag = z + f64(b), mag + f64(b).abs()
    y = act(z, activation)
    # A sum of I products in any order: I roundings of at most 2^-24 of the magnitudes.  The slopes of the
    # activations stay under 1.13; each is good to a few units of its own value and argument.
    bound = (x.shape[-1] + 8) * 2.0 ** -24 * 1.13 * mag + 16 * 2.0 ** -24 * y.abs()
    if residual is not None:
        y = y + f64(residual)
        bound = bound + 2.0 ** -24 * y.abs()
    return y, bound


def norm_rope(x, weight, positions, cos, sin, eps, rms, interleaved):
    z = f64(x)
    if rms:
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    if weight is not None:
        z = z * f64(weight)
    if cos is None:
        return z, z.abs()
    half = cos.shape[1]
    out, mag = z.clone(), z.abs()
    p = torch.tensor(positions, dtype=torch.int64)
    there = (p >= 0) & (p < cos.shape[0])
    c, s = (f64(t)[torch.where(there, p, 0)][:, None, :] for t in (cos, sin))
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    a, b = z[..., first], z[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    mag[..., first] = mag[..., second] = a.abs() + b.abs()
    out[~there] = float("nan")
    return out, mag


def e4m3(t):
    """Nearest e4m3 number, ties to even, of a float64 array within +-448."""
    t = np.asarray(t, dtype=np.float64)
    _, e = np.frexp(np.abs(t))
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.rint(t / step) * step


def code(x, scale, fmt):
    """Numbers (before the scale) of fp32 values x in a block of fp32 scale."""
    q = np.float32(x) / np.float32(scale)
    q = np.where(np.isnan(q), np.float32(0), q)
    q = np.clip(q, -QMAX[fmt], QMAX[fmt]).astype(np.float64)
    return np.rint(q) if fmt == "int8" else e4m3(q)


class Cache:
    """The cache's definition, one page and head at a time."""

    def __init__(self, pages, heads, dim, page, fmt):
        self.codes = {n: np.zeros((pages, heads, page, dim)) for n in "kv"}
        self.scales = {n: np.zeros((pages, heads), dtype=np.float32) for n in "kv"}
        self.pages, self.page, self.fmt = pages, page, fmt

    def write(self, k, v, table, starts, offsets):
        for name, src in (("k", k), ("v", v)):
            x = src.float().cpu().numpy()
            for b in range(len(starts)):
                n, first = offsets[b + 1] - offsets[b], starts[b]
                if n == 0:
                    continue
                for p0 in range(first // self.page * self.page, first + n, self.page):
                    if p0 // self.page >= len(table[b]):
                        continue
                    g = table[b][p0 // self.page]
                    if not 0 <= g < self.pages:
                        continue
                    r0, r1 = max(first - p0, 0), min(first + n - p0, self.page)
                    new = x[offsets[b] + p0 + r0 - first:offsets[b] + p0 + r1 - first]
                    for h in range(x.shape[1]):
                        self._block(name, g, h, r0, r1, new[:, h])

    def _block(self, name, g, h, r0, r1, new):
        finite = np.where(np.isfinite(new), np.abs(new), np.float32(0))
        scale = np.float32(max(np.float32(finite.max()) / np.float32(QMAX[self.fmt]), np.float32(2.0 ** -100)))
        codes, old = self.codes[name][g, h], self.scales[name][g, h]
        if r0 > 0:
            scale = max(scale, old)
            if scale != old:
                codes[:r0] = code(np.float32(codes[:r0]) * old, scale, self.fmt)
        codes[r0:r1] = code(new, scale, self.fmt)
        self.scales[name][g, h] = scale

    def value(self, name, table, b, p):
        """[heads][dim] in 64 bits, or None where there is no page."""
        if p < 0 or p // self.page >= len(table[b]):
            return None
        g = table[b][p // self.page]
        if not 0 <= g < self.pages:
            return None
        return self.codes[name][g, :, p % self.page] * self.scales[name][g].astype(np.float64)[:, None]


def attention(q, cache, table, lengths, offsets, causal, window, scale):
    """(y, p|v|, |s|, p scale): the result, the weights' sum over the values' magnitudes, the largest
    sum of magnitudes behind a row's scores, and a row's largest weight times its block's value scale."""
    q = f64(q).numpy()
    t, hq, dim = q.shape
    y, mag, smag, top = np.zeros(q.shape), np.zeros(q.shape), np.zeros((t, hq, 1)), np.zeros((t, hq, 1))
    for b in range(len(lengths)):
        n = offsets[b + 1] - offsets[b]
        keys = [(j, cache.value("k", table, b, j), cache.value("v", table, b, j)) for j in range(lengths[b])]
        keys = [e for e in keys if e[1] is not None]
        if not keys or n == 0:
            continue
        pos = np.array([e[0] for e in keys])
        k, v = np.stack([e[1] for e in keys]), np.stack([e[2] for e in keys])
        vs = np.stack([cache.scales["v"][table[b][j // cache.page]] for j in pos]).astype(np.float64)
        group = hq // k.shape[1]
        for i in range(n):
            p = lengths[b] - n + i
            seen = np.ones(len(pos), bool)
            if causal:
                seen &= pos <= p
            if window:
                seen &= pos > p - window
            if not seen.any():
                continue
            for h in range(hq):
                kk, vv = k[seen][:, h // group], v[seen][:, h // group]
                row = q[offsets[b] + i, h]
                s = kk @ row * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                y[offsets[b] + i, h] = w @ vv
                mag[offsets[b] + i, h] = w @ np.abs(vv)
                top[offsets[b] + i, h] = (w * vs[seen][:, h // group]).max()
                smag[offsets[b] + i, h] = (np.abs(kk) @ np.abs(row)).max() * abs(scale)
    return y, mag, smag, top


def attention_bound(y, mag, smag, top, dim, dtype):
    """Error that a kernel of the stated precision stays within: its output's
    rounding; weights held in 11 bits (bf16 outputs) or 22 (fp32); the roundings
    of the scores' sums (dim + 8 of them, and an exponential good to a few
    units of its argument), which move every weight by twice as much; and the
    smallest step of a weight, 2^-39 of the row's largest weight times its
    block's value scale (`top`): half of it for each of up to 2^10 keys with
    codes up to 2^9, 2^-21 of `top`."""
    weight = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    score = (dim + 16) * 2.0 ** -24 * smag
    return half_ulp(dtype) * np.abs(y) + (weight + 2 * score + 2.0 ** -20) * mag + 2.0 ** -21 * top + 1e-37
