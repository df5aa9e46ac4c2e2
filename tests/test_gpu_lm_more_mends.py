"""GPU checks of single properties of prompt attention, linear layers on codes and
logit adjustments, each at the calls where it can be lost."""
import numpy as np
import pytest
import torch

import ref_lm as ref
import ref_lm_more as more
import ref_prompt_bits as bits
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2410_08300_amd as cs  # noqa: E402
from test_gpu_lm_more import DEV, DT, check_prompt, close, gen, heads_of, ints  # noqa: E402


# ---- prompt attention -------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128, 200])
@pytest.mark.parametrize("seqs,n", [(64, 3), (40, 300), (5, 300), (2, 450)])  # 128, 64 and 32 rows a workgroup
def test_prompt_holds_its_weights_in_24_bits(dtype, dim, seqs, n):
    say("case prompt bits", dtype, dim, seqs, n,
        cs.describe_prompt_attention(seqs, seqs * n, 16, 8, dim, DT[dtype], causal=False))
    q, k, v, offsets, w, places = bits.cancelling(dim + n, seqs, n, 8, dim, DT[dtype])
    want, mag = bits.result(v, w, places, n)
    q = q.repeat_interleave(2, 1)  # two heads to a key head
    y = cs.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), ints(offsets), causal=False, scale=1.0)
    every = lambda t: t[:, None].expand(-1, n, -1, -1).reshape(seqs * n, 8, dim).repeat_interleave(2, 1)  # noqa: E731
    close(y, every(want), every(bits.bound(want, mag, DT[dtype])), "bits")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [32, 128, 256])
@pytest.mark.parametrize("counts", [[2, 1, 5], [400, 150], [300] * 16], ids=str)
def test_prompt_averages_values_near_the_largest_number(dtype, dim, counts):
    """An average lies among its values; their sum leaves fp32 from the second one on."""
    say("case prompt large values", dtype, dim, counts)
    q, k, v = heads_of(gen(dim), sum(counts), 4, 2, dim, DT[dtype], fused=False)
    v = (torch.sign(v.float()) * 3.2e38 * (0.5 + torch.sigmoid(v.float()) / 2)).to(DT[dtype])
    v[:, 0] = v[:, 0].abs()
    y = check_prompt(q, k, v, counts)
    assert bool(torch.isfinite(y).all())
    check_prompt(q, k, v, counts, True, 40)
    v[counts[0] - 1, 0, 3] = float("-inf")  # reaches the rows that see it, which is one
    check_prompt(q, k, v, counts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -133, -2.0 ** -130, 2.0 ** -126])
def test_prompt_scales_below_the_least_normal_number(dtype, scale):
    """Scores of up to 2^126 times such scales are small, and at a scale of zero all weights are alike."""
    q, k, v = heads_of(gen(7), 200, 4, 2, 16, DT[dtype], fused=False)
    q = torch.full_like(q, 2.0 ** 60)
    k = (2.0 ** 62 * torch.sigmoid(k.float())).to(DT[dtype])
    check_prompt(q, k, v, [120, 80], True, 0, scale)


def test_prompt_scale_of_the_largest_size():
    q, k, v = heads_of(gen(8), 60, 2, 1, 32, torch.float32, fused=False)
    check_prompt(q * 2.0 ** -60, k * 2.0 ** -68, v, [60], True, 0, 2.0 ** 127)


@pytest.mark.parametrize("n,dim,causal,window", bits.F32_CASES)
def test_prompt_in_fp32_is_as_near_as_fp32_steps(n, dim, causal, window):
    say("case prompt fp32", n, dim, causal, window)
    q, k, v = bits.f32_case(n, dim)
    want = more.prompt(q, k, v, [0, n], causal, window, dim ** -0.5)[0]
    limit = 2 * bits.far(bits.plain_f32(q, k, v, causal, window, dim ** -0.5), want)
    for copies in (1, 2, 14):  # 32 to 128 rows a workgroup
        y = cs.prompt_attention(*(t.repeat(copies, 1, 1).to(DEV) for t in (q, k, v)),
                                ints([n * i for i in range(copies + 1)]), causal=causal, window=window)
        for part in y.split(n):
            found = bits.far(part, want)
            assert bool((found <= limit).all()), (found, limit)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offsets,like", [
    ([0, 100], [0, 64]), ([-5, 30, 64], [0, 30, 64]), ([0, 20, 2 ** 31 - 1], [0, 20, 64]), ([70, 80], None),
    ([-2 ** 31, -1], None), ([0, 50, 20, 64], []), ([2 ** 31 - 1, -2 ** 31, 5], []), ([64, 0], [])], ids=str)
def test_prompt_offsets_outside_the_tokens(offsets, like, dtype):
    """Clamped to the tokens; nothing beside the result is written, and what does not rise may give anything there."""
    say("case prompt offsets", offsets, dtype)
    q, k, v = heads_of(gen(6), 64, 4, 2, 32, DT[dtype], fused=False)
    held = torch.full((64 + 2 * 200, 4, 32), 7.0, dtype=DT[dtype], device=DEV)
    out = held[200:264]
    cs.prompt_attention(q, k, v, ints(offsets), out=out)
    assert bool((held[:200] == 7).all()) and bool((held[264:] == 7).all())
    if like is None:
        assert bool((out == 7).all())
    elif like:
        assert torch.equal(out, cs.prompt_attention(q, k, v, ints(like)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,dim,window", [([5003], 64, 0), ([4097, 1000], 128, 3000), ([6000], 32, 5500)], ids=str)
def test_prompt_of_thousands_of_tokens(dtype, counts, dim, window):
    say("case prompt long", dtype, counts, dim, window)
    q, k, v = heads_of(gen(sum(counts)), sum(counts), 2, 1, dim, DT[dtype])
    check_prompt(q, k, v, counts, True, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_beyond_one_launch(dtype):
    """More sequences than a launch's third axis holds: one token each, whose result is its value, to three roundings in
    fp32: of the value times a weight near one, of one over that weight (their only sum), and of the product of both.
    bf16's own rounding takes them back."""
    say("case prompt launches", dtype)
    n = 140001
    q, k, v = heads_of(gen(1), n + 90, 2, 1, 32, DT[dtype])
    offsets = torch.arange(n + 2, device=DEV, dtype=torch.int32)
    offsets[-1] = n + 90
    y = cs.prompt_attention(q, k, v, offsets)
    off = (y[:n].double() - v[:n].double()).abs()
    assert bool((off <= (3.01 * 2.0 ** -24 if dtype == "f32" else 0) * v[:n].double().abs()).all())
    want, mag, smag = more.prompt(q[n:], k[n:], v[n:], [0, 90], True, 0, 32 ** -0.5)
    close(y[n:], want, more.prompt_bound(want, mag, smag, 90, 32, DT[dtype]), "last")


@pytest.mark.parametrize("dtype,es", [("bf16", 2), ("f32", 4)])
def test_prompt_rows_as_far_apart_as_a_tile_reaches(dtype, es):
    """The last rows of a tile lie 2 GiB behind its first; rows further apart are copied."""
    say("case prompt strides", dtype)
    near = 2 ** 31 // 128 // es - 256
    q, k, v = heads_of(gen(2), 150, 4, 2, 64, DT[dtype], fused=False)
    for step in (near, near + 256):
        held = torch.empty(149 * step + 2 * 128, dtype=DT[dtype], device=DEV)
        kk = torch.as_strided(held, (150, 2, 64), (step, 128, 1))
        vv = torch.as_strided(held, (150, 2, 64), (step, 128, 1), 64)
        kk.copy_(k), vv.copy_(v)
        check_prompt(q, kk, vv, [150])
        check_prompt(q, kk, vv, [21, 129], False)


# ---- codes ------------------------------------------------------------------------

def powers(g, n, low, high):
    """n scales spread over 2^low .. 2^high."""
    e = low + (high - low) * torch.rand(n, generator=g, dtype=torch.float64)
    return torch.exp2(e).float()


# One and several rows through registers, and tiles of 64, of 128, of 256, and of parts that are joined.
@pytest.mark.parametrize("m,i,o", [(1, 64, 40), (3, 200, 35), (70, 64, 260), (2048, 128, 6144), (4090, 1024, 4090),
                                   (64, 16384, 320)])
@pytest.mark.parametrize("low,high", [(-149, -20), (-60, 0), (-100, 100), (0, 127)])
def test_int8_results_of_scales_far_apart(m, i, o, low, high):
    """What a sum and two scales give in fp32 is right to its last bits wherever fp32 holds it, whatever the scales'
    product: a sum's conversion, two products of numbers near one and, below 2^-126, the place of the last bit."""
    say("case int8 scales", m, i, o, low, high, cs.describe_linear_int8(m, i, o, torch.float32, True))
    g = torch.Generator().manual_seed(m + i + o)
    x, w = (torch.randint(-128, 128, (n, i), generator=g, dtype=torch.int8) for n in (m, o))
    xs = powers(g, m, low, high)
    # Results within fp32 and beside its ends: scales of the outputs are the others' reciprocals, more or less.
    ws = powers(g, o, max(-149, -90 - high), min(127, -20 - low))
    y = cs.linear_int8(x.to(DEV), w.to(DEV), ws.to(DEV), x_scale=xs.to(DEV), dtype=torch.float32)
    want = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()[None]
    most = torch.finfo(torch.float32).max
    near = (want.abs() / most - 1).abs() < 2.0 ** -20  # on either side of infinity
    want = torch.where(near, 0.0, torch.where(want.abs() > most, want * np.inf, want))
    y = torch.where(near, 0.0, y.cpu())
    close(y, want, 3.01 * 2.0 ** -24 * want.abs() + 2.0 ** -149, "scales")


# ---- logits -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype,n,vocab", [("bf16", 260, 200003), ("f32", 130, 200003), ("bf16", 120, 70001),
                                           ("f32", 120, 70001), ("bf16", 512, 500)])
@pytest.mark.parametrize("seen", [40, 4100])
def test_logits_of_every_width_and_store(dtype, n, vocab, seen):
    """Results of more than 96 MiB go past the caches; rows are those of one alone, on any alignment."""
    say("case logits stores", dtype, n, vocab, seen)
    x = torch.randn(n, vocab, generator=gen(n), device=DEV).to(DT[dtype])
    h = torch.randint(0, vocab, (n * seen,), generator=gen(1), device=DEV, dtype=torch.int32)
    off = torch.arange(n + 1, device=DEV, dtype=torch.int32) * seen
    p = [0.5 + torch.rand(n, generator=gen(2 + i), device=DEV) for i in range(3)]
    mask = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=gen(9), device=DEV).to(torch.int32)
    whole = cs.adjust_logits(x, h, off, None, *p, mask=mask)
    for b in (0, 1, n // 2, n - 1):
        one = cs.adjust_logits(x[b:b + 1], h[b * seen:(b + 1) * seen], ints([0, seen]), None, *(t[b:b + 1] for t in p),
                               mask=mask[b:b + 1])
        assert torch.equal(whole[b], one[0])
    want, mag = more.logits(x[n - 1:], h[-seen:].tolist(), [0, seen], None, *(t[n - 1:] for t in p), None, mask[n - 1:])
    size = torch.where(torch.isfinite(want), want.abs(), 0.0)
    close(whole[n - 1:], want, 6 * 2.0 ** -24 * mag + 1.01 * ref.half_ulp(x.dtype) * size + 1e-37, "stores")


# ---- more than 2^31 values ----------------------------------------------------------

def test_prompt_of_more_than_32_bits_of_values():
    say("case prompt beyond 2^31 values")
    n, count = 530000, 265
    q = torch.randn(n, 32, 128, generator=gen(3), device=DEV, dtype=torch.bfloat16)
    k, v = q.roll(1, 1), q.roll(2, 1)
    offsets = torch.arange(n // count + 1, device=DEV, dtype=torch.int32) * count
    y = cs.prompt_attention(q, k, v, offsets)
    for at in (0, n // 2 // count * count, n - count):
        part = [t[at:at + count, 30:].clone() for t in (q, k, v)]
        want, mag, smag = more.prompt(*part, [0, count], True, 0, 128 ** -0.5)
        close(y[at:at + count, 30:], want, more.prompt_bound(want, mag, smag, count, 128, torch.bfloat16), "far")


@pytest.mark.parametrize("m,i,o", [(70000, 64, 32768), (40000, 64, 60002)])
def test_int8_of_more_than_32_bits_of_values(m, i, o):
    say("case int8 beyond 2^31 values", m, i, o)
    g = gen(4)
    x = torch.randint(-128, 128, (m, i), generator=g, device=DEV, dtype=torch.int8)
    w = torch.randint(-128, 128, (o, i), generator=g, device=DEV, dtype=torch.int8)
    xs, ws = torch.rand(m, generator=g, device=DEV), torch.rand(o, generator=g, device=DEV) * 1e-3
    y = cs.linear_int8(x, w, ws, x_scale=xs)
    for rows in (slice(0, 3), slice(m // 2, m // 2 + 3), slice(m - 3, m)):  # sums are whole numbers: the same bits
        assert torch.equal(y[rows], cs.linear_int8(x[rows], w, ws, x_scale=xs[rows]))
    codes, scales = cs.quantize_rows(y)
    for rows in (slice(0, 3), slice(m - 3, m)):
        want, wanted = more.quantize(y[rows])
        assert np.array_equal(codes[rows].cpu().numpy(), want) and np.array_equal(scales[rows].cpu().numpy(), wanted)


def test_logits_of_more_than_32_bits_of_values():
    say("case logits beyond 2^31 values")
    n, vocab = 17000, 128001
    x = torch.randn(n, vocab, generator=gen(5), device=DEV, dtype=torch.bfloat16)
    h = torch.randint(0, vocab, (n * 20,), generator=gen(6), device=DEV, dtype=torch.int32)
    off = torch.arange(n + 1, device=DEV, dtype=torch.int32) * 20
    p = [0.5 + torch.rand(n, generator=gen(7 + i), device=DEV) for i in range(3)]
    mask = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=gen(9), device=DEV).to(torch.int32)
    y = cs.adjust_logits(x, h, off, None, *p, mask=mask)
    for b in (0, n // 2, n - 1):
        one = cs.adjust_logits(x[b:b + 1], h[b * 20:b * 20 + 20], ints([0, 20]), None, *(t[b:b + 1] for t in p),
                               mask=mask[b:b + 1])
        assert torch.equal(y[b], one[0])
