"""The measured work of the language-model operators: the pieces of a decoder
layer served from a cache held in 8 bits.

A case is one pass through one operator:

* ``linear``: ``linear(x, w, b, act, residual)``, the matrix product of a layer
  with its bias, activation and residual add;
* ``qk_norm_rope``: ``qk_norm_rope(q, k, ...)``, the RMS norm of every query and
  key head and its position rotation, on the two slices of a fused projection;
* ``cache``: ``KVCache.write`` of new tokens, which quantises them in blocks of
  one page and head, then ``KVCache.read`` of the tokens as values;
* ``attention``: ``cached_attention``, new queries over such a cache.

``own`` false computes the same from elementary torch operations in 32 bits;
``exact`` does so in 64, written apart.  A stored code is a discrete decision, so
the operators define it by its 32-bit steps (a block's scale is a stored 32-bit
number, and codes come from the 32-bit quotient), and all three follow them.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ES = {"f32": 4, "bf16": 2}
_QMAX = {"int8": 127.0, "fp8": 448.0}
_MIN_SCALE = 2.0 ** -100

# A drawn case does no more work than the largest listed ones.
_MAX_FLOPS = {"linear": {"bf16": 5.4e11, "f32": 5.0e10}, "attention": {"bf16": 1.3e11, "f32": 3.0e10}}
_MAX_BYTES = 1.0e9


def _linear(name, dtype, m, i, o, act, bias, residual):
    return {"name": name, "op": "linear", "dtype": dtype, "m": m, "in": i, "out": o, "act": act, "bias": bias,
            "residual": residual}


def _rope(name, dtype, tokens, q_heads, kv_heads, dim, rotary, interleaved, weight):
    return {"name": name, "op": "qk_norm_rope", "dtype": dtype, "tokens": tokens, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "interleaved": interleaved, "weight": weight}


def _cache(name, dtype, fmt, seqs, new, past, ragged, kv_heads, dim, page, read):
    return {"name": name, "op": "cache", "dtype": dtype, "fmt": fmt, "seqs": seqs, "new": new, "past": past,
            "ragged": ragged, "kv_heads": kv_heads, "dim": dim, "page": page, "read": read}


def _attn(name, dtype, fmt, seqs, new, past, ragged, q_heads, kv_heads, dim, page, window, causal=True):
    return {"name": name, "op": "attention", "dtype": dtype, "fmt": fmt, "seqs": seqs, "new": new, "past": past,
            "ragged": ragged, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "page": page, "window": window,
            "causal": causal}


def listed():
    return [
        # A projection of one token being generated, with the residual it is added to: weight-bound, latency counts.
        _linear("linear_1x4096x4096_bf16", "bf16", 1, 4096, 4096, "none", False, True),
        # The widening product of a feed-forward layer over a long prompt, with bias and activation: matrix-bound.
        _linear("linear_4096x4096x16384_bf16", "bf16", 4096, 4096, 16384, "gelu_tanh", True, False),
        # A classifier on a ragged batch in fp32: the headline network's 2048 features, sizes that no tile divides.
        _linear("linear_333x2048x1001_f32", "f32", 333, 2048, 1001, "relu", True, False),
        # Queries and keys of one generated token of one sequence: latency alone.
        _rope("rope_1_bf16", "bf16", 1, 32, 8, 128, 128, False, True),
        # ... and of a batch of long prompts: traffic.
        _rope("rope_16384_bf16", "bf16", 16384, 32, 8, 128, 128, False, True),
        # fp32 with neighbours rotated as pairs, part of a head rotated, an odd number of tokens and heads of 80.
        _rope("rope_1021_f32", "f32", 1021, 12, 12, 80, 32, True, False),
        # One generated token of each of 64 sequences goes into pages that are partly full (their scales may grow).
        _cache("cache_64x1_int8", "bf16", "int8", 64, 1, 4000, True, 8, 128, 16, "touched"),
        # Prompts of unlike lengths go into an empty cache, and are read back whole.
        _cache("cache_6x4096_fp8", "bf16", "fp8", 6, 4096, 0, True, 8, 128, 64, "all"),
        # One generated token of one sequence over a long context: few rows, a long axis.
        _attn("attention_1x1_32768_int8", "bf16", "int8", 1, 1, 32767, False, 32, 8, 128, 64, 0),
        # One generated token of each of 64 sequences of unlike lengths: the traffic of serving.
        _attn("attention_64x1_8192_fp8", "bf16", "fp8", 64, 1, 8191, True, 32, 8, 128, 16, 0),
        # The prompt of a long document, causal: matrix-bound.
        _attn("attention_1x4096_int8", "bf16", "int8", 1, 4096, 0, False, 32, 8, 128, 64, 0),
        # fp32 chunks of prompts of odd lengths behind a cached prefix, in a sliding window, heads of 80.
        _attn("attention_3x301_f32", "f32", "int8", 3, 301, 700, True, 12, 4, 80, 32, 513),
    ]


# ---- drawn cases -----------------------------------------------------------

def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Feature counts: mostly multiples of 8 or 64, some of any size (never 3072, a kernel-benchmark size)."""
    v = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64, 64))
    v = v if v < 2 * step else v // step * step
    return v + 8 if v == 3072 else v


def _heads(rng):
    kv = rng.choice((1, 2, 3, 4, 8, 8, 16))
    return kv * rng.choice((1, 2, 3, 4, 4, 8)), kv


def draw(rng):
    op = rng.choice(("linear", "linear", "qk_norm_rope", "cache", "attention", "attention"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 192, 256))
    while True:
        q_heads, kv_heads = _heads(rng)
        if op == "linear":
            case = _linear("", dtype, _log(rng, 1, 8192), _width(rng, 48, 16384), _width(rng, 48, 16384),
                           rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), rng.random() < 0.5,
                           rng.random() < 0.5)
        elif op == "qk_norm_rope":
            case = _rope("", dtype, _log(rng, 1, 16384), q_heads, kv_heads, dim,
                         rng.choice((dim, dim, dim // 2, dim // 4)), rng.random() < 0.5, rng.random() < 0.7)
        else:
            fmt, page = rng.choice(("int8", "fp8")), rng.choice((16, 32, 64, 128))
            seqs = _log(rng, 1, 128)
            new = 1 if rng.random() < 0.5 else _log(rng, 1, 4096)
            past = 0 if rng.random() < 0.2 else _log(rng, 1, 32768)
            ragged = seqs > 1 and rng.random() < 0.8
            if op == "cache":
                case = _cache("", dtype, fmt, seqs, new, past, ragged, kv_heads, dim, page,
                              rng.choice(("touched", "all")))
            else:
                window = 0 if rng.random() < 0.7 else _log(rng, 8, 4096)
                case = _attn("", dtype, fmt, seqs, new, past, ragged, q_heads, kv_heads, dim, page, window,
                             rng.random() < 0.85)
        w = work(case)
        if w["bytes"] <= _MAX_BYTES and w["flops"] <= _MAX_FLOPS.get(op, {}).get(dtype, 1e12):
            # What the cache of a case holds stays within what its own largest listed case holds.
            if op in ("linear", "qk_norm_rope") or sum(_lengths(case)[1]) * kv_heads * dim <= 3.0e8:
                del case["name"]
                return case


# ---- inputs ----------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens cached before them) of every sequence, as whole numbers."""
    n = case["seqs"]
    if not case["ragged"]:
        return [case["new"]] * n, [case["past"]] * n
    # Lengths between a quarter of the case's and all of it, spread by a golden-ratio walk.
    f = [0.25 + 0.75 * ((i * 0.6180339887498949 + 0.37) % 1.0) for i in range(n)]
    return [max(1, round(case["new"] * v)) for v in f], [round(case["past"] * v) for v in f]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)


def _layout(case, gen):
    """Block table of a paged cache whose pages were handed out in no order, and the host lengths."""
    new, past = _lengths(case)
    ps = case["page"]
    total = [a + b for a, b in zip(new, past)]
    need = [(t + ps - 1) // ps for t in total]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int64)
    width = max(need)
    table = torch.full((len(need), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].to(torch.int32)
        at += n
    return {"new": new, "past": past, "total": total, "pages": pages, "table": table}


def _offsets(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _kv(case, tokens, gen):
    """Keys and values as projections give them: a few strong key channels, values of uneven head scales."""
    h, d = case["kv_heads"], case["dim"]
    dt = _DT[case["dtype"]]
    chan = 1.0 + 3.0 * (torch.rand(h, d, generator=gen, device="cuda") < 0.03)
    k = (torch.randn(tokens, h, d, generator=gen, device="cuda") * chan).to(dt)
    v = (torch.randn(tokens, h, d, generator=gen, device="cuda")
         * (0.25 + torch.rand(h, 1, generator=gen, device="cuda"))).to(dt)
    return k, v


def prepare(case, seed):
    gen = _generator(seed)
    dt = _DT[case["dtype"]]
    s = {"case": case}
    if case["op"] == "linear":
        m, i, o = case["m"], case["in"], case["out"]
        s["x"] = torch.randn(m, i, generator=gen, device="cuda").to(dt)
        s["w"] = (torch.randn(o, i, generator=gen, device="cuda") * (2.0 / i) ** 0.5).to(dt)
        s["b"] = (torch.randn(o, generator=gen, device="cuda") * 0.1).to(dt) if case["bias"] else None
        s["r"] = torch.randn(m, o, generator=gen, device="cuda").to(dt) if case["residual"] else None
        return s
    if case["op"] == "qk_norm_rope":
        t, hq, hk, d, rot = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"], case["rotary"]
        # The fused projection's rows: queries, keys and values side by side.
        s["qkv"] = (torch.randn(t, (hq + 2 * hk) * d, generator=gen, device="cuda") * 1.7).to(dt)
        s["q"] = s["qkv"][:, :hq * d].view(t, hq, d)
        s["k"] = s["qkv"][:, hq * d:(hq + hk) * d].view(t, hk, d)
        s["qw"] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) if case["weight"] else None
        s["kw"] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) if case["weight"] else None
        limit = 32768
        s["positions"] = torch.randint(0, limit, (t,), generator=gen, device="cuda", dtype=torch.int32)
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        angle = torch.arange(limit, device="cuda", dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        return s
    lay = _layout(case, gen)
    s.update(lay)
    h, d, ps, fmt = case["kv_heads"], case["dim"], case["page"], case["fmt"]
    s["cu"] = torch.tensor(_offsets(lay["new"]), dtype=torch.int32, device="cuda")
    s["past_dev"] = torch.tensor(lay["past"], dtype=torch.int32, device="cuda")
    s["total_dev"] = torch.tensor(lay["total"], dtype=torch.int32, device="cuda")
    # What is in the cache at the call: the past, and for attention the new tokens too.
    filled = lay["past"] if case["op"] == "cache" else lay["total"]
    zero = torch.zeros(case["seqs"], dtype=torch.int32, device="cuda")
    k, v = _kv(case, sum(filled), gen)
    plain = {"k": torch.zeros(lay["pages"], h, ps, d, device="cuda", dtype=_code_dtype(fmt)),
             "v": torch.zeros(lay["pages"], h, ps, d, device="cuda", dtype=_code_dtype(fmt)),
             "ks": torch.zeros(lay["pages"], h, device="cuda"), "vs": torch.zeros(lay["pages"], h, device="cuda")}
    if own:
        import paper_2410_08300_amd as cs
        s["cache"] = cs.KVCache(lay["pages"], h, d, page_size=ps, fmt=fmt)
        if k.shape[0]:
            cu = torch.tensor(_offsets(filled), dtype=torch.int32, device="cuda")
            s["cache"].write(k, v, lay["table"], zero, cu)
    else:
        _plain_write(plain, k, v, lay["table"], [0] * case["seqs"], filled, fmt)
        s["plain"] = plain
    if case["op"] == "cache":
        s["k"], s["v"] = _kv(case, sum(lay["new"]), gen)
        s["from"] = [p // ps * ps if case["read"] == "touched" else 0 for p in lay["past"]]
        counts = [t - f for t, f in zip(lay["total"], s["from"])]
        s["read_counts"] = counts
        s["from_dev"] = torch.tensor(s["from"], dtype=torch.int32, device="cuda")
        s["read_cu"] = torch.tensor(_offsets(counts), dtype=torch.int32, device="cuda")
    else:
        sharp = 1.0 + 2.0 * torch.rand(case["q_heads"], 1, generator=gen, device="cuda")
        s["q"] = (torch.randn(sum(lay["new"]), case["q_heads"], d, generator=gen, device="cuda") * sharp).to(dt)
    return s


# ---- the operators in their plain form -----------------------------------------

def _plain_act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.7071067811865476))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_linear(s):
    y = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        y = y + s["b"].float()
    y = _plain_act(y, s["case"]["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(s["x"].dtype)


def _plain_rope(s):
    rot, inter = s["case"]["rotary"], s["case"]["interleaved"]
    pos = s["positions"].long()
    cos, sin = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        z = x.float()
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + 1e-6)
        if w is not None:
            z = z * w.float()
        r = z[..., :rot]
        a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
        lo, hi = a * cos - b * sin, b * cos + a * sin
        r = torch.stack((lo, hi), -1).flatten(-2) if inter else torch.cat((lo, hi), -1)
        out.append(torch.cat((r, z[..., rot:]), -1).to(x.dtype))
    return out


def _code_dtype(fmt):
    return torch.int8 if fmt == "int8" else torch.float8_e4m3fn


def _encode(x, scale, fmt):
    t = x / scale
    if fmt == "int8":
        return torch.round(t).clamp(-127, 127).to(torch.int8)
    return t.clamp(-448, 448).to(torch.float8_e4m3fn)


def _plain_write(c, k, v, table, past, counts, fmt):
    """New tokens into their pages: a page's scale covers its largest magnitude, never shrinks while the page
    fills, and what the page held is coded again when it grows."""
    ps = c["k"].shape[2]
    # On the device: torch divides by a host number by multiplying with its reciprocal, which rounds otherwise.
    qmax = torch.full((), _QMAX[fmt], device=k.device)
    at = 0
    for b, n in enumerate(counts):
        if n == 0:
            continue
        p0, end = past[b] // ps, (past[b] + n + ps - 1) // ps
        pages = table[b, p0:end].long()
        lead = past[b] - p0 * ps
        for codes, scales, new in ((c["k"], c["ks"], k), (c["v"], c["vs"], v)):
            h, d = new.shape[1:]
            x = torch.zeros((end - p0) * ps, h, d, device=new.device)
            x[lead:lead + n] = new[at:at + n].float()
            x = x.view(end - p0, ps, h, d).permute(0, 2, 1, 3)
            scale = (x.abs().amax((2, 3)) / qmax).clamp(min=_MIN_SCALE)
            if lead:
                old_scale = scales[pages[0]].clone()
                scale[0] = torch.maximum(scale[0], old_scale)
                old = codes[pages[0], :, :lead].float() * old_scale[:, None, None]
                x = x.contiguous()
                x[0, :, :lead] = old
            q = _encode(x, scale[:, :, None, None], fmt)
            tail = past[b] + n - (end - 1) * ps
            if tail < ps:
                q[-1, :, tail:] = codes[pages[-1], :, tail:]
            codes[pages] = q
            scales[pages] = scale
        at += n


def _plain_gather(c, name, pages):
    """Values [tokens][heads][dim] of whole pages."""
    codes, scales = c[name], c[name + "s"]
    x = codes[pages].float() * scales[pages][:, :, None, None]
    return x.permute(0, 2, 1, 3).flatten(0, 1)


def _plain_cache(s):
    case = s["case"]
    ps, dt = case["page"], _DT[case["dtype"]]
    _plain_write(s["plain"], s["k"], s["v"], s["table"], s["past"], s["new"], case["fmt"])
    out = []
    for name in ("k", "v"):
        parts = []
        for b, n in enumerate(s["read_counts"]):
            p0 = s["from"][b] // ps
            pages = s["table"][b, p0:(s["total"][b] + ps - 1) // ps].long()
            parts.append(_plain_gather(s["plain"], name, pages)[:n])
        out.append(torch.cat(parts).to(dt))
    return out


def _plain_attention(s):
    case = s["case"]
    hq, h, d, ps = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(s["q"].shape, device="cuda", dtype=s["q"].dtype)
    at = 0
    for b, n in enumerate(s["new"]):
        t = s["total"][b]
        pages = s["table"][b, :(t + ps - 1) // ps].long()
        k = _plain_gather(s["plain"], "k", pages)[:t].permute(1, 2, 0).contiguous()
        v = _plain_gather(s["plain"], "v", pages)[:t].permute(1, 0, 2).contiguous()
        q = s["q"][at:at + n].float().view(n, h, hq // h, d).permute(1, 2, 0, 3).reshape(h, hq // h * n, d)
        z = torch.matmul(q, k).view(h, hq // h, n, t) * (1.0 / math.sqrt(d))
        i = torch.arange(t - n, t, device="cuda")[:, None]
        j = torch.arange(t, device="cuda")[None, :]
        hide = torch.zeros(n, t, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hide |= j > i
        if case["window"]:
            hide |= j <= i - case["window"]
        z = z.masked_fill(hide, float("-inf"))
        z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
        total = z.sum(-1, keepdim=True)
        z = z / torch.where(total > 0, total, torch.ones_like(total))
        y = torch.matmul(z.view(h, hq // h * n, t), v)
        out[at:at + n] = y.view(h, hq // h, n, d).permute(2, 0, 1, 3).reshape(n, hq, d).to(out.dtype)
        at += n
    return out


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"linear": _plain_linear, "qk_norm_rope": _plain_rope, "cache": _plain_cache,
                "attention": _plain_attention}[op](state)
    import paper_2410_08300_amd as cs
    if op == "linear":
        return cs.linear(state["x"], state["w"], state["b"], act=case["act"], residual=state["r"])
    if op == "qk_norm_rope":
        return cs.qk_norm_rope(state["q"], state["k"], state["positions"], state["cos"], state["sin"],
                               q_weight=state["qw"], k_weight=state["kw"], eps=1e-6,
                               interleaved=case["interleaved"])
    if op == "cache":
        state["cache"].write(state["k"], state["v"], state["table"], state["past_dev"], state["cu"])
        return state["cache"].read(state["table"], state["from_dev"], state["read_cu"], sum(state["read_counts"]),
                                   dtype=_DT[case["dtype"]])
    return cs.cached_attention(state["q"], state["cache"], state["table"], state["total_dev"], state["cu"],
                               causal=case["causal"], window=case["window"])


# ---- work ------------------------------------------------------------------

def _pairs(case):
    """Query-key pairs that the masks leave, and keys that some query of their sequence sees."""
    new, past = _lengths(case)
    pairs = keys = 0
    for n, p in zip(new, past):
        t, w = n + p, case["window"] or n + p
        if not case["causal"]:
            # Row i sees (i - w, t).
            pairs += sum(t - max(0, p + i - w + 1) for i in range(n))
        else:
            pairs += sum(min(p + i + 1, w) for i in range(n))
        keys += t - max(0, p - w + 1)
    return pairs, keys


def work(case):
    es = _ES[case["dtype"]]
    if case["op"] == "linear":
        m, i, o = case["m"], case["in"], case["out"]
        return {"bytes": es * (m * i + o * i + m * o * (2 if case["residual"] else 1) + (o if case["bias"] else 0)),
                "flops": 2 * m * i * o}
    if case["op"] == "qk_norm_rope":
        heads = case["q_heads"] + case["kv_heads"]
        t, d = case["tokens"], case["dim"]
        return {"bytes": t * (2 * heads * d * es + 4 + 4 * case["rotary"]) + (2 * d * es if case["weight"] else 0),
                "flops": t * heads * (4 * d + 3 * case["rotary"])}
    new, past = _lengths(case)
    h, d, ps = case["kv_heads"], case["dim"], case["page"]
    if case["op"] == "cache":
        start = [p // ps * ps if case["read"] == "touched" else 0 for p in past]
        written, read = sum(new), sum(n + p - f for n, p, f in zip(new, past, start))
        return {"bytes": 2 * h * d * (written * (es + 1) + read * (es + 1)), "flops": 2 * h * d * (3 * written + read)}
    pairs, keys = _pairs(case)
    return {"bytes": 2 * keys * h * d + 8 * h * (keys // ps) + 2 * sum(new) * case["q_heads"] * d * es,
            "flops": 4 * pairs * case["q_heads"] * d}


# ---- the definitions in 64 bits ----------------------------------------------

def _exact_linear(s):
    # Rows in blocks: the product's 64-bit operands need not all be there at once.
    case, w = s["case"], s["w"].double()
    parts = []
    for lo in range(0, s["x"].shape[0], 1024):
        z = torch.matmul(s["x"][lo:lo + 1024].double(), w.transpose(0, 1))
        if s["b"] is not None:
            z += s["b"].double()
        if case["act"] == "relu":
            z = torch.where(z > 0, z, torch.zeros_like(z))
        elif case["act"] == "gelu":
            z = z * torch.special.ndtr(z)
        elif case["act"] == "gelu_tanh":
            # (1 + tanh u) / 2 is the logistic function of 2 u.
            z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        elif case["act"] == "silu":
            z = z * torch.sigmoid(z)
        if s["r"] is not None:
            z = z + s["r"][lo:lo + 1024].double()
        parts.append(z)
    return torch.cat(parts)


def _exact_rope(s):
    case, outs = s["case"], []
    rot, pos = case["rotary"], s["positions"].long()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[pos].unsqueeze(1)
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        z = x.double()
        z = z / torch.sqrt(z.pow(2).sum(-1, keepdim=True) / z.shape[-1] + 1e-6)
        if w is not None:
            z = z * w.double()
        y = z.clone()
        first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
        second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)
        c = torch.complex(z[..., first], z[..., second]) * turn
        y[..., first], y[..., second] = c.real, c.imag
        outs.append(y)
    return outs


def _exact_code(x, scale, fmt):
    """The number a code stands for before its scale, from the 32-bit quotient."""
    t = (x.double() / scale.double()).float().double()
    if fmt == "int8":
        return t.round().clamp(-127, 127)
    # Four significant bits, the smallest step 2^-9.
    _, e = torch.frexp(t.abs())
    step = (((e.long() - 4).clamp(min=-9) + 1023) << 52).view(torch.float64)
    return ((t / step).round() * step).clamp(-448, 448)


def _exact_fill(x, past_codes, past_scale, fmt):
    """Codes and scale of one block after tokens x [n][d] follow the codes it holds ([m][d] or None)."""
    scale = (x.double().abs().amax() / _QMAX[fmt]).clamp(min=_MIN_SCALE).float()
    if past_codes is None:
        return _exact_code(x, scale, fmt), scale
    scale = torch.maximum(scale, past_scale)
    held = (past_codes * past_scale.double()).float()
    return torch.cat((_exact_code(held, scale, fmt), _exact_code(x, scale, fmt))), scale


def _exact_blocks(x, ps, fmt):
    """Values of a sequence written at once from its first position: [tokens][heads][dim] in 64 bits."""
    n, h, d = x.shape
    full = (n + ps - 1) // ps
    y = torch.zeros(full * ps, h, d, device=x.device, dtype=torch.float64)
    y[:n] = x.double()
    y = y.view(full, ps, h, d)
    scale = (y.abs().amax((1, 3), keepdim=True) / _QMAX[fmt]).clamp(min=_MIN_SCALE).float()
    return (_exact_code(y, scale, fmt) * scale.double()).view(full * ps, h, d)[:n], scale.view(full, h)


def _exact_inputs(case, seed):
    """The inputs that prepare makes, without a cache: float keys and values in the order they are written."""
    gen = _generator(seed)
    lay = _layout(case, gen)
    filled = lay["past"] if case["op"] == "cache" else lay["total"]
    k, v = _kv(case, sum(filled), gen)
    return gen, lay, filled, k, v


def _exact_cache(case, seed):
    gen, lay, filled, k0, v0 = _exact_inputs(case, seed)
    k1, v1 = _kv(case, sum(lay["new"]), gen)
    ps, fmt, h = case["page"], case["fmt"], case["kv_heads"]
    outs = []
    for old, new in ((k0, k1), (v0, v1)):
        parts, oat, nat = [], 0, 0
        for n, p in zip(lay["new"], lay["past"]):
            before, after = old[oat:oat + p], new[nat:nat + n]
            oat, nat = oat + p, nat + n
            whole, lead = p // ps * ps, p % ps
            rows = []
            if whole and case["read"] == "all":
                rows.append(_exact_blocks(before[:whole], ps, fmt)[0])
            first = min(n, ps - lead) if lead else 0
            if lead:
                heads = []
                for i in range(h):
                    held, hs = _exact_fill(before[whole:, i], None, None, fmt)
                    codes, scale = _exact_fill(after[:first, i], held, hs, fmt)
                    heads.append(codes * scale.double())
                rows.append(torch.stack(heads, 1))
            if n > first:
                rows.append(_exact_blocks(after[first:], ps, fmt)[0])
            parts.append(torch.cat(rows))
        outs.append(torch.cat(parts))
    return outs


def _exact_attention(case, seed):
    gen, lay, _, k, v = _exact_inputs(case, seed)
    sharp = 1.0 + 2.0 * torch.rand(case["q_heads"], 1, generator=gen, device="cuda")
    q = (torch.randn(sum(lay["new"]), case["q_heads"], case["dim"], generator=gen, device="cuda") * sharp)
    q = q.to(_DT[case["dtype"]]).double()
    group, parts, at, kat = case["q_heads"] // case["kv_heads"], [], 0, 0
    for n, t in zip(lay["new"], lay["total"]):
        kk = _exact_blocks(k[kat:kat + t], case["page"], case["fmt"])[0]
        vv = _exact_blocks(v[kat:kat + t], case["page"], case["fmt"])[0]
        row = torch.arange(n, device="cuda").unsqueeze(1) + (t - n)
        col = torch.arange(t, device="cuda").unsqueeze(0)
        seen = torch.ones(n, t, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen &= col <= row
        if case["window"]:
            seen &= row - col < case["window"]
        heads = []
        for hq in range(case["q_heads"]):
            z = torch.matmul(q[at:at + n, hq], kk[:, hq // group].transpose(0, 1)) / math.sqrt(case["dim"])
            z = torch.softmax(torch.where(seen, z, torch.full_like(z, float("-inf"))), -1)
            z = torch.where(seen.any(1, keepdim=True), z, torch.zeros_like(z))
            heads.append(torch.matmul(z, vv[:, hq // group]))
        parts.append(torch.stack(heads, 1))
        at, kat = at + n, kat + t
    return torch.cat(parts)


def exact(case, seed):
    if case["op"] == "linear":
        return _exact_linear(prepare(case, seed))
    if case["op"] == "qk_norm_rope":
        return _exact_rope(prepare(case, seed))
    if case["op"] == "cache":
        return _exact_cache(case, seed)
    return _exact_attention(case, seed)
