"""Plain 64-bit CPU forms of prompt attention, linear layers on codes and logit
adjustments, written from their definitions in include/convsel_lm.h, with the
magnitudes that bound a kernel's error."""
import math

import numpy as np
import torch

import ref_lm as ref


def prompt(q, k, v, offsets, causal, window, scale):
    """(y, sum of weights times the values' magnitudes, largest sum of magnitudes behind a row's scores); y is NaN in
    rows that belong to no sequence."""
    q, k, v = ref.f64(q), ref.f64(k), ref.f64(v)
    t, hq, dim = q.shape
    group = hq // k.shape[1]
    y = torch.full((t, hq, dim), float("nan"), dtype=torch.float64)
    mag, smag = torch.zeros(t, hq, dim, dtype=torch.float64), torch.zeros(t, hq, 1, dtype=torch.float64)
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        n = hi - lo
        i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
        seen = (j <= i) if causal else torch.ones(n, n, dtype=torch.bool)
        if window:
            seen = seen & (j > i - window)
        for h in range(hq):
            kk, vv, qq = k[lo:hi, h // group], v[lo:hi, h // group], q[lo:hi, h]
            s = torch.where(seen, qq @ kk.T * scale, -math.inf)
            p = torch.softmax(s, 1)
            # What is hidden has no part in the sums, whatever it holds.
            clean = torch.where(torch.isfinite(vv), vv, 0.0)
            out = p @ clean
            odd = ~torch.isfinite(vv)
            if odd.any():
                for r, c in odd.nonzero().tolist():
                    out[seen[:, r], c] += vv[r, c]
            y[lo:hi, h] = out
            mag[lo:hi, h] = p @ clean.abs()
            if n:
                m = torch.where(seen, qq.abs() @ kk.abs().T, 0.0) * abs(scale)
                smag[lo:hi, h, 0] = m.max(1).values
    return y, mag, smag


def prompt_bound(y, mag, smag, n, dim, dtype):
    """The output's rounding; the scores' sums, of dim products, and their scale and exponential, which move every
    weight by twice as much; weights in 16 bits or more (bf16) or 24; and sums over n keys of weights and of products,
    each rounded, of two parts in bf16."""
    weight = 2.0 ** -17 if dtype == torch.bfloat16 else 0.0
    score = (dim + 16) * 2.0 ** -24 * smag
    return ref.half_ulp(dtype) * y.abs() + (weight + 2 * score + (4 * n + 16) * 2.0 ** -24 + 2.0 ** -19) * mag + 1e-37


def quantize(x):
    """(codes, scales) of rows, by the definition's fp32 steps."""
    x = x.detach().float().cpu().numpy()
    finite = np.where(np.isfinite(x), np.abs(x), np.float32(0))
    scale = np.maximum(finite.max(-1) / np.float32(127), np.float32(2.0 ** -100)).astype(np.float32)
    with np.errstate(all="ignore"):
        q = x / scale[..., None]
    q = np.where(np.isnan(q), np.float32(0), q)
    return np.rint(np.clip(q, -127, 127)).astype(np.int8), scale


def linear_int8(codes, scale, w, w_scale, b, activation, residual):
    """(y, bound): three roundings of the scaled sum, one of the bias, the activation's slope (under 1.13) and its own
    few units, and the residual's."""
    codes, w = (torch.as_tensor(t.astype(np.float64)) for t in (codes, w))
    acc = codes @ w.T  # whole numbers below 2^53
    z = acc * torch.as_tensor(scale).double()[..., None] * torch.as_tensor(w_scale).double()
    mag = z.abs()
    if b is not None:
        z, mag = z + ref.f64(b), mag + ref.f64(b).abs()
    y = ref.act(z, activation)
    bound = 5 * 2.0 ** -24 * 1.13 * mag + 16 * 2.0 ** -24 * y.abs()
    if residual is not None:
        y = y + ref.f64(residual)
        bound = bound + 2.0 ** -24 * y.abs()
    return y, bound


def logits(x, history, offsets, prompts, rep, pres, freq, bias, mask):
    """(y, magnitudes that four fp32 roundings may show)."""
    z = ref.f64(x)
    mag = z.abs()
    n, vocab = z.shape
    for b in range(n):
        if history is not None:
            tokens = [t for t in history[offsets[b]:offsets[b + 1]]]
            lead = prompts[b] if prompts is not None else 0
            for t in set(tokens):
                if not 0 <= t < vocab:
                    continue
                if rep is not None:
                    r = float(rep[b])
                    z[b, t] = z[b, t] / r if z[b, t] > 0 else z[b, t] * r
                made = tokens[lead:].count(t)
                less = 0.0
                if made:
                    less = float(freq[b]) * made if freq is not None else 0.0
                    less += float(pres[b]) if pres is not None else 0.0
                mag[b, t] = max(mag[b, t], abs(z[b, t])) + abs(less)
                z[b, t] -= less
        if bias is not None:
            row = ref.f64(bias) if bias.dim() == 1 else ref.f64(bias)[b]
            z[b] += row
            mag[b] += row.abs()
        if mask is not None:
            words = (mask if mask.dim() == 1 else mask[b]).tolist()
            allowed = torch.tensor([(words[t // 32] >> (t % 32)) & 1 for t in range(vocab)], dtype=torch.bool)
            z[b] = torch.where(allowed, z[b], -math.inf)
    return z, mag
