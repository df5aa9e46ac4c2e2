"""GPU checks of single properties of the decoder operators, each at the calls
where it can be lost: how many bits a result keeps, scales of zero, numbers that
leave a type, outputs beside inputs, and sizes at the end of a range."""
import numpy as np
import pytest
import torch

import ref_lm as ref
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2410_08300_amd as cs  # noqa: E402
from test_gpu_lm import DEV, DT, build, fresh, gen, ints, offsets_of, wide, within  # noqa: E402


# ---- attention: bits ----------------------------------------------------------

def half_step(y, dtype):
    """Half the distance between neighbours of the type around |y|."""
    bits = 8 if dtype == torch.bfloat16 else 24
    _, e = np.frexp(np.maximum(np.abs(y), 1e-30))
    return np.ldexp(0.5, e - bits)


@pytest.mark.parametrize("kernel", ["rows", "tiles"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_differs_from_its_definition_by_the_last_rounding(dtype, fmt, kernel):
    """Scores here are whole multiples of 2^-5 that fp32 sums hold exactly: keys are small whole numbers in pages of
    scale one, queries multiples of 1/4.  What is left before the output's own rounding: the score's factor (three
    roundings of it, |s| up to 12: 52 units of 2^-24 in the exponent of 2), its place under the maximum (a rounding of
    up to 48: as much again), the exponential (4), the weight's two halves (2^-22: 4 units) and the sum of 64 products
    and of 64 weights (64 each), with up to 2^-20 (16) between blocks: under 256 units, 2^-16 of the weighted
    magnitudes."""
    say("case attention bits", dtype, fmt, kernel)
    hq, hk, dim, page = 8, 2, 64, 16
    lengths = [64, 50, 33]
    new = [2, 1, 1] if kernel == "rows" else [64, 50, 33]
    g, dt = gen(77), DT[dtype]
    table = [[4, 0, 9, 2], [7, 3, 10, 5], [1, 8, 6, -1]]
    cache, want = fresh(12, hk, dim, page, fmt)
    off, zeros = offsets_of(lengths), [0, 0, 0]
    k = torch.randint(-8, 9, (off[-1], hk, dim), generator=g, device=DEV).to(dt)
    k[:, :, 0] = ref.QMAX[fmt]  # the block's scale is one; no query looks at this column
    v = torch.randn(off[-1], hk, dim, generator=g, device=DEV).to(dt)
    cache.write(k, v, ints(table), ints(zeros), ints(off))
    want.write(k, v, table, zeros, off)
    assert bool((cache.k_scales[[4, 0, 9, 2, 7, 3, 10, 5, 1, 8, 6]] == 1).all())
    q = (torch.randint(-1, 2, (sum(new), hq, dim), generator=g, device=DEV) * 0.25).to(dt)
    q[:, :, 0] = 0
    scale = 0.125
    t = ints(table) if kernel == "rows" else wide(table, (hq, hk, dim, page, lengths, new))
    text = cs.describe_attention(cache, 3, sum(new), t.shape[1], hq, dt)
    assert "attention_%s_kernel" % kernel in text, text
    y = cs.cached_attention(q, cache, t, ints(lengths), ints(offsets_of(new)), scale=scale)
    exact, mag, smag, top = ref.attention(q, want, table, lengths, offsets_of(new), True, 0, scale)
    assert smag.max() <= 12
    before = 2.0 ** -16 * mag
    within(y, exact, before + half_step(np.abs(exact) + before, dt), "bits %s %s %s" % (dtype, fmt, kernel))


# ---- attention: scales of zero ----------------------------------------------------

def planned(kernel, case, table, dtype):
    """(times that the sequences are repeated, table) that bring a call to the kernel named, "rows", "128" or "256"."""
    hq, hk, dim, page, lengths, new = case[:6]
    if kernel == "rows":
        rep, t = 1, ints(table)
    elif kernel == "128" and dtype == "bf16":
        rep = int(2e9 / (sum(new) * hq * len(table[0]) * page * ((dim + 31) // 32 * 32))) + 1
        t = ints(table)
    else:
        rep, t = 1, wide(table, case)
    t = t.repeat(rep, 1)
    text = cs.describe_attention(_Shape(hk, dim, page), len(new) * rep, sum(new) * rep, t.shape[1], hq, DT[dtype])
    assert " rows=%s " % (16 if kernel == "rows" else kernel) in text, text
    return rep, t


class _Shape:
    """What describe_attention reads of a cache: its sizes."""

    def __init__(self, kv_heads, head_dim, page):
        self._cache = cs.KVCache(1, kv_heads, head_dim, page_size=page)
        self._desc, self.head_dim = self._cache._desc, head_dim


ZERO_CASE = (4, 1, 64, 16, [400, 63, 200, 17], [130, 40, 200, 20], True, 0)


@pytest.mark.parametrize("kernel,dtype", [("rows", "bf16"), ("rows", "f32"), ("128", "bf16"), ("128", "f32"), ("256", "bf16")])
def test_attention_over_pages_that_nothing_was_written_to(kernel, dtype):
    """A new cache holds zeros in pages of scale zero, and a warm-up call reads them: the result is zero.  Among written
    pages, of values so small that a scale of one beside them would leave their weights no bits, such pages count with
    their scores (zero keys) and add zeros."""
    say("case attention zero scales", kernel, dtype)
    hq, hk, dim, page, lengths, new = ZERO_CASE[:6]
    small = [2, 2, 2, 2] if kernel == "rows" else new
    case = ZERO_CASE[:5] + (small, True, 0)
    for what in ("all", "one", "tiny"):
        cache, want, table, q = build(case, "int8", dtype, seed=8)
        if what == "all":
            cache = cs.KVCache(cache.pages, hk, dim, page_size=page)
            for s in want.scales.values():
                s[:] = 0
        else:
            gain = np.float32(1.0 if what == "one" else 1e-9)
            cache.v_scales.mul_(float(gain))
            want.scales["v"] *= gain
            for b, i in ((0, 3), (1, 0), (2, 1), (2, 12), (3, 0)):  # one that a causal mask hides from whole waves
                cache.v_scales[table[b][i], 0] = 0
                want.scales["v"][table[b][i], 0] = 0
                cache.k_scales[table[b][i], 0] = 0
                want.scales["k"][table[b][i], 0] = 0
        rep, t = planned(kernel, case, table, dtype)
        offs = [0]
        for _ in range(rep):
            offs += [offs[-1] + o for o in offsets_of(small)[1:]]
        y = cs.cached_attention(q.repeat(rep, 1, 1), cache, t, ints(lengths * rep), ints(offs)).view(rep, -1, hq, dim)
        exact, mag, smag, top = ref.attention(q, want, table, lengths, offsets_of(small), True, 0, 0.125)
        within(y[0], exact, ref.attention_bound(exact, mag, smag, top, dim, q.dtype), "zero scales %s" % what)
        assert bool((y == y[0]).all())
        if what == "all":
            assert bool((y == 0).all())


# ---- cache: its buffers -------------------------------------------------------------

@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_cache_scales_are_fp32_under_any_default_type(default):
    say("case cache default type", default)
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        cache = cs.KVCache(8, 2, 32, page_size=16)
    finally:
        torch.set_default_dtype(before)
    for s in (cache.k_scales, cache.v_scales):
        assert s.dtype == torch.float32 and s.shape == (8, 2)
    want = ref.Cache(8, 2, 32, 16, "int8")
    x = torch.randn(100, 2, 32, generator=gen(1), device=DEV)
    table, off = [[7, 6, 5, 4, 3, 2, 1]], [0, 100]
    cache.write(x, x, ints(table), ints([0]), ints(off))
    want.write(x, x, table, [0], off)
    assert np.array_equal(cache.k_scales.cpu().numpy()[1:], want.scales["k"][1:])


@pytest.mark.parametrize("name", ["k_codes", "v_codes", "k_scales", "v_scales"])
def test_cache_buffers_take_values_and_no_other_tensor(name):
    """The library holds their addresses: another tensor in their place would leave it with freed memory."""
    cache = cs.KVCache(4, 2, 32)
    held = getattr(cache, name)
    with pytest.raises(AttributeError, match="cannot be replaced"):
        setattr(cache, name, held.clone())
    assert getattr(cache, name) is held
    held.copy_(torch.ones_like(held))
    cache.k_scales *= 2
    cache.v_scales += 1
    assert bool((held != 0).all()) and getattr(cache, name) is held


def test_attention_windows_of_more_than_32_bits_hide_nothing():
    case = (4, 2, 64, 16, [60], [3], True, 0)
    cache, _, table, q = build(case, "int8", "bf16")
    args = (q, cache, ints(table), ints([60]), ints([0, 3]))
    y = cs.cached_attention(*args)
    assert not torch.equal(cs.cached_attention(*args, window=8), y)
    for window in (2 ** 31 - 1, 2 ** 32 + 8, 2 ** 63 - 1):
        assert torch.equal(cs.cached_attention(*args, window=window), y)
    with pytest.raises((ValueError, cs.Conv2dError)):
        cs.cached_attention(*args, window=-2 ** 32 + 8)


# ---- linear: the end of its range ---------------------------------------------------

def test_linear_of_more_rows_than_a_launch_has_tiles_of_64():
    """2^30 rows and one, of eight outputs: 17 GB in and out."""
    m = 2 ** 30 + 1
    say("case linear", m, cs.describe_linear(m, 8, 8))
    x = torch.zeros(m, 8, dtype=torch.bfloat16, device=DEV)
    w = torch.randn(8, 8, generator=gen(2), device=DEV).bfloat16()
    rows = torch.tensor([0, 1, 255, 256, 2 ** 29, 2 ** 30 - 1, 2 ** 30], device=DEV)
    x[rows] = torch.randn(len(rows), 8, generator=gen(3), device=DEV).bfloat16()
    y = cs.linear(x, w)
    want, bound = ref.linear(x[rows], w)
    within(y[rows], want, bound + ref.half_ulp(torch.bfloat16) * want.abs() * 1.01, "many rows")
    y[rows] = 0
    assert not any(bool(part.any()) for part in y.split(2 ** 26))


# ---- linear: activations far left of zero ---------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
def test_activations_keep_their_precision_where_they_are_small(activation, dtype):
    """Relative to the result, in units of 2^-24.  gelu in fp32: the fit 0.3, its sum of nine terms up to three times
    their total 27, t's two roundings 8, the exponential, its correction and four products 8: 48.  silu: the exponential's
    argument is exact (bf16 multiplies it by log2 e: its rounding and the constant's), a few operations: 16 + 3 |z|.
    gelu_tanh: six roundings of the exponential's argument u and a few operations: 16 + 8 |u|.  In bf16 gelu's exponent
    has the roundings of z^2 and of log2 e times half of it, and one more in the constant: 64 + 2 z^2."""
    say("case activation tails", activation, dtype)
    dt, low = DT[dtype], {"gelu": -12.5, "gelu_tanh": -9.0, "silu": -80.0}[activation]
    z = torch.cat([torch.linspace(low, 0, 20001, device=DEV), torch.linspace(0, 12, 2001, device=DEV)]).to(dt)[:, None]
    y = cs.linear(z, torch.ones(1, 1, device=DEV, dtype=dt), act=activation)
    a = ref.f64(z).abs()
    if activation == "gelu":
        want = ref.act(ref.f64(z), "gelu")  # by erfc, which does not cancel
        units = 48.0 if dtype == "f32" else 64 + 2 * a ** 2
    elif activation == "gelu_tanh":
        want = ref.f64(z) * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (ref.f64(z) + 0.044715 * ref.f64(z) ** 3))
        units = 16 + 8 * 1.6 * (a + 0.044715 * a ** 3)
    else:
        want = ref.f64(z) * torch.sigmoid(ref.f64(z))
        units = 16 + 3 * a
    before = units * 2.0 ** -24 * want.abs() + 1e-36
    within(y, want, before + torch.from_numpy(half_step((want.abs() + before).numpy(), dt)), "%s %s" % (activation, dtype))


# ---- sequences of very unlike lengths --------------------------------------------------

@pytest.mark.parametrize("rows,dtype,dim", [(16, "bf16", 32), (16, "f32", 32), (256, "bf16", 32), (128, "f32", 32),
                                            (128, "bf16", 160)])
def test_long_sequences_among_many_short_ones(rows, dtype, dim):
    """150 sequences, most of one new token, some of none (the first and the last too), two of many: written, read back
    and attended in one call each.  Every workgroup has to find the sequence that its tile is of."""
    say("case unlike", rows, dtype, dim)
    g, dt, hq, hk, page, seqs = gen(dim), DT[dtype], 16, 1, 16, 150
    new, held = [1] * seqs, [(7 * b) % 41 for b in range(seqs)]
    for b in (0, 1, 50, 51, 52, 120, 149):
        new[b] = 0
    new[40], new[121], held[40] = 300, 70, 23
    total = [h + n for h, n in zip(held, new)]
    need = [(t + page - 1) // page for t in total]
    order, at, table = torch.randperm(sum(need) + 2, generator=g, device=DEV).tolist(), 0, []
    for n in need:
        table.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    cache, want = fresh(sum(need) + 2, hk, dim, page, "int8")
    zeros = [0] * seqs
    for starts, counts in ((zeros, held), (held, new)):
        off = offsets_of(counts)
        k, v = (torch.randn(off[-1], hk, dim, generator=g, device=DEV).to(dt) for _ in range(2))
        cache.write(k, v, ints(table), ints(starts), ints(off))
        want.write(k, v, table, starts, off)
    off = offsets_of(total)
    for got, name in zip(cache.read(ints(table), ints(zeros), ints(off), off[-1], dtype=torch.float32), "kv"):
        exact = np.concatenate([np.stack([want.value(name, table, b, p) for p in range(n)])
                                for b, n in enumerate(total) if n]).astype(np.float32)
        assert np.array_equal(got.cpu().numpy(), exact), name
    q = torch.randn(sum(new), hq, dim, generator=g, device=DEV).to(dt)
    t = ints(table) if rows == 16 else wide(table, (hq, hk, dim, page, total, new))
    text = cs.describe_attention(cache, seqs, sum(new), t.shape[1], hq, dt)
    assert " rows=%d " % rows in text, text
    # Tokens behind the last offset are nobody's, and stay as they are.
    whole = torch.full((sum(new) + 5, hq, dim), 7.0, device=DEV, dtype=dt)
    more = torch.cat([q, q[:5]])
    cs.cached_attention(more, cache, t, ints(total), ints(offsets_of(new)), out=whole)
    exact, mag, smag, top = ref.attention(q, want, table, total, offsets_of(new), True, 0, dim ** -0.5)
    within(whole[:-5], exact, ref.attention_bound(exact, mag, smag, top, dim, dt), "unlike")
    assert bool((whole[-5:] == 7).all())


def test_more_sequences_than_a_grids_third_axis_holds():
    """70001 sequences of one or two tokens and one of 3000, in one call each.  Keys and values are whole numbers up to
    127, exact in their pages; a sequence's first query sees its first token alone."""
    seqs, long = 70001, 68000
    say("case many sequences", seqs)
    new = torch.ones(seqs, dtype=torch.int64, device=DEV)
    new[::2] = 2
    new[long] = 3000
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), new.cumsum(0)])
    tokens = int(off[-1])
    table = torch.full((seqs, 188), -1, dtype=torch.int32, device=DEV)
    table[:, 0] = torch.arange(seqs, device=DEV)
    table[long, 1:] = torch.arange(seqs, seqs + 187, device=DEV)
    cache = cs.KVCache(seqs + 187, 1, 16)
    k, v = (torch.randint(-127, 128, (tokens, 1, 16), generator=gen(s), device=DEV).bfloat16() for s in (1, 2))
    k[:, :, 0] = v[:, :, 0] = 127
    off, zeros, lengths = off.int(), torch.zeros(seqs, dtype=torch.int32, device=DEV), new.int()
    cache.write(k, v, table, zeros, off)
    k2, v2 = cache.read(table, zeros, off, tokens)
    assert torch.equal(k2, k) and torch.equal(v2, v)
    q = torch.randn(tokens, 2, 16, generator=gen(3), device=DEV).bfloat16()
    y = cs.cached_attention(q, cache, table, lengths, off)
    first = off[:-1].long()
    assert torch.equal(y[first], v[first].expand(-1, 2, -1))
    assert bool(y.isfinite().all())


# ---- the example ------------------------------------------------------------------------

def test_decoder_example_refuses_prompts_that_it_has_no_next_token_for():
    """An empty prompt has no last token whose logits could be its own."""
    from test_gpu_decoder import SMALL, decoder
    model = decoder.Decoder(**SMALL)
    for prompts, new in (([[], [1, 2]], 3), ([[1, 2], []], 3), ([], 3), ([[1]], 0)):
        with pytest.raises(ValueError, match="at least"):
            model.generate(prompts, new)
    assert model.generate([[1], [2, 3]], 1)[0].shape == (2, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 12, 100, 400])
def test_linear_carries_infinities_of_both_signs_in_their_own_rows(m, dtype):
    """An infinity of x meets weights of either sign (and no zeros): its row is infinite, each output with its weight's
    sign, and both infinities in one row leave NaN where their products differ in sign."""
    g, dt = gen(m), DT[dtype]
    x = torch.randn(m, 320, generator=g, device=DEV).to(dt)
    w = torch.randn(200, 320, generator=g, device=DEV).to(dt)
    w[w == 0] = 1
    clean = cs.linear(x, w)
    row, inf = m // 2, float("inf")
    keep = torch.arange(m, device=DEV) != row
    for places in ({5: inf}, {319: -inf}, {0: inf, 200: inf}, {7: inf, 311: -inf}):
        bad = x.clone()
        for k, v in places.items():
            bad[row, k] = v
        y = cs.linear(bad, w)
        assert torch.equal(y[keep], clean[keep])
        signs = torch.stack([w[:, k].sign() * (1 if v > 0 else -1) for k, v in places.items()])
        same = (signs == signs[0]).all(0)
        want = torch.where(same, signs[0] * inf, torch.full_like(signs[0], float("nan")))
        assert torch.equal(torch.nan_to_num(y[row], nan=7.0), torch.nan_to_num(want, nan=7.0)), places


@pytest.mark.parametrize("seqs,at", [(600, 0), (600, 300), (600, 599), (40, 17)])
def test_one_sequence_with_tokens_among_idle_ones(seqs, at):
    """A batch of fixed places of which one has a prompt, of no more tokens than there are places.  Whole numbers up to
    127 are exact in their pages; the first query sees the first token alone."""
    n = seqs - 3
    say("case idle", seqs, at)
    counts = [0] * seqs
    counts[at] = n
    off = ints(offsets_of(counts))
    pages = (n + 5 + 15) // 16
    table = torch.full((seqs, pages), -1, dtype=torch.int32, device=DEV)
    table[at] = torch.arange(pages, device=DEV).flip(0)
    starts, lengths = torch.zeros_like(off[:-1]), ints(counts)
    cache = cs.KVCache(pages, 2, 32)
    k, v = (torch.randint(-127, 128, (n, 2, 32), generator=gen(s), device=DEV).bfloat16() for s in (1, 2))
    k[:, :, 0] = v[:, :, 0] = 127
    for start in (0, 5):  # from a page's first row, and from within one: as many tokens reach a page more
        starts[at], lengths[at] = start, start + n
        cache.write(k, v, table, starts, off)
        k2, v2 = cache.read(table, starts, off, n)
        assert torch.equal(k2, k) and torch.equal(v2, v), start
        q = torch.randn(n, 4, 32, generator=gen(3), device=DEV).bfloat16()
        y = cs.cached_attention(q, cache, table, lengths, off)
        assert bool(y.isfinite().all())
        if start == 0:
            assert torch.equal(y[0], v[0].repeat_interleave(2, 0))
