"""Prompt attention, linear layers on 8-bit codes and logit adjustments against
plain 64-bit forms, at the sizes, strides and masks where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2410_08300_amd as cs
import ref_lm as ref
import ref_lm_more as more
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = torch.device("cuda")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def offsets_of(counts):
    return [0] + list(np.cumsum(counts))


def close(got, want, bound, what):
    """Every value within its bound; what is not finite is the same."""
    got, want = ref.f64(got), want.double()
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)]), what
    err = torch.where(odd, 0.0, (got - want).abs())
    bad = err > bound
    assert not bool(bad.any()), "%s: %d of %d, worst %.3g of its bound" % (
        what, int(bad.sum()), bad.numel(), float((err / bound)[~odd].max()))


# ---- prompt attention -----------------------------------------------------------

def heads_of(g, t, hq, hk, dim, dtype, fused=True):
    sharp = 1 + 2 * torch.rand(hq, 1, generator=g, device=DEV)
    q, k, v = randn(g, t, hq, dim) * sharp, randn(g, t, hk, dim), randn(g, t, hk, dim)
    rows = torch.cat((q, k, v), 1).to(dtype)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())


def check_prompt(q, k, v, counts, causal=True, window=0, scale=None, **kw):
    offsets = offsets_of(counts)
    dim = q.shape[2]
    s = 1 / math.sqrt(dim) if scale is None else scale
    y = cs.prompt_attention(q, k, v, ints(offsets), causal=causal, window=window, scale=scale, **kw)
    n = offsets[-1]
    want, mag, smag = more.prompt(q, k, v, offsets, causal, window, s)
    close(y[:n], want[:n], more.prompt_bound(want, mag, smag, max(counts), dim, q.dtype)[:n], "prompt")
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [1, 8, 20, 32, 40, 64, 80, 96, 127, 128, 160, 192, 224, 256])
def test_prompt_head_widths(dtype, dim):
    say("case prompt width", dtype, dim)
    q, k, v = heads_of(gen(dim), 206, 4, 2, dim, DT[dtype])
    check_prompt(q, k, v, [70, 1, 0, 135])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1], [2], [31], [32, 33], [63, 64, 65], [127, 128, 129], [1] * 40, [0, 0, 5, 0],
                                    [513], [300, 1, 1, 1, 1, 1, 1, 1, 200]], ids=str)
@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 8), (6, 2), (16, 1)])
def test_prompt_lengths_and_groups(dtype, counts, hq, hk):
    say("case prompt lengths", dtype, counts, hq, hk)
    q, k, v = heads_of(gen(sum(counts) + hq), sum(counts), hq, hk, 64, DT[dtype], fused=hq != 8)
    check_prompt(q, k, v, counts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 2, 31, 64, 100, 129, 2 ** 31 + 5])
def test_prompt_masks(dtype, causal, window):
    say("case prompt masks", dtype, causal, window)
    q, k, v = heads_of(gen(window % 1000), 400, 3, 3, 48, DT[dtype])
    check_prompt(q, k, v, [261, 7, 132], causal, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3, 4.0])
def test_prompt_scales(dtype, scale):
    say("case prompt scale", dtype, scale)
    q, k, v = heads_of(gen(3), 150, 4, 2, 32, DT[dtype])
    check_prompt(q, k, v, [150], True, 0, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,causal", [(0, True), (70, True), (40, False)])
def test_prompt_hidden_values_have_no_influence(dtype, window, causal):
    """Infinities and NaN in keys and values reach the rows that see them, and no other."""
    say("case prompt hidden", dtype, window, causal)
    q, k, v = heads_of(gen(9), 400, 4, 2, 64, DT[dtype], fused=False)
    counts = [190, 200]  # and ten rows of no sequence
    v[100, 0, 3], v[100, 1, 63], v[150, 0, 5] = float("inf"), float("nan"), -float("inf")
    v[189, 0], v[200, 1, 10], v[389, 1] = float("nan"), float("inf"), -float("inf")
    v[390:], k[390:], q[390:] = float("nan"), float("nan"), float("nan")
    out = torch.full_like(q, 7.0)
    y = check_prompt(q, k, v, counts, causal, window, out=out)
    assert y is out and bool((out[390:] == 7).all())
    # A key that is NaN makes a row's softmax NaN where it is seen.
    k[60, 0, 0] = float("nan")
    y = cs.prompt_attention(q, k, v, ints(offsets_of(counts)), causal=causal, window=window)
    i = torch.arange(190, device=DEV)
    sees = (i >= 60) if causal else torch.ones_like(i, dtype=torch.bool)
    if window:
        sees &= i - 60 < window
    assert bool(torch.isnan(y[:190, :2][sees]).all()) and not bool(torch.isnan(y[:100, :2][~sees[:100]]).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_strides_and_alignments(dtype):
    """Rows on no 16 bytes, odd strides, a broadcast head, transposed layouts, and an output between others."""
    say("case prompt strides", dtype)
    g, dt = gen(5), DT[dtype]
    base = randn(g, 90, 4 * 70 + 1, dtype=dt)
    q, k, v = base[:, 1:129].view(90, 2, 64), base[:, 129:193].view(90, 1, 64), base[:, 193:257].view(90, 1, 64)
    check_prompt(q, k, v, [50, 40])
    q, k, v = heads_of(g, 90, 4, 4, 64, dt, fused=False)
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    check_prompt(*turned, [50, 40])
    check_prompt(q, k[:, :1].expand(-1, 4, -1), v[:, 1:2].expand(-1, 4, -1), [50, 40])
    check_prompt(q, k[:1].expand(90, -1, -1), v[:1].expand(90, -1, -1), [50, 40])
    wide = torch.full((90, 4, 67), 3.0, dtype=dt, device=DEV)
    check_prompt(q, k, v, [50, 40], out=wide[:, :, 1:65])
    assert bool((wide[:, :, :1] == 3).all()) and bool((wide[:, :, 65:] == 3).all())


def test_prompt_offsets_are_bounded():
    """Offsets that do not rise or leave the tokens are clamped: no row of another call's memory is touched."""
    q, k, v = heads_of(gen(6), 64, 2, 1, 32, torch.bfloat16, fused=False)
    for offsets in ([0, 100], [-5, 30, 64], [0, 50, 20, 64], [70, 80], [2 ** 31 - 1, -2 ** 31, 5]):
        y = cs.prompt_attention(q, k, v, ints(offsets))
        torch.cuda.synchronize()
        assert y.shape == q.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [40, 64, 128, 200])
@pytest.mark.parametrize("rows,counts", [(128, [301] * 14), (64, [370] * 5 + [1, 0, 7]), (32, [450, 400])])
def test_prompt_rows_of_a_workgroup(dtype, dim, rows, counts):
    """Waves that share out rows, keys, or both."""
    say("case prompt rows", dtype, dim, rows)
    assert "rows=%d " % rows in cs.describe_prompt_attention(len(counts), sum(counts), 16, 8, dim, DT[dtype]) or (
        dim == 200 and rows == 32)
    q, k, v = heads_of(gen(rows + dim), sum(counts), 16, 8, dim, DT[dtype])
    check_prompt(q, k, v, counts)
    check_prompt(q, k, v, counts, True, 77)
    v[counts[0] - 40, 2, 5] = float("inf")
    k[20, 1, 0] = k[20, 1, 0] * 0 + 60
    check_prompt(q, k, v, counts)


def test_prompt_repeats_bit_for_bit_and_long_rows_agree_with_many_heads():
    q, k, v = heads_of(gen(8), 2000, 8, 2, 128, torch.bfloat16)
    off = ints([0, 1300, 2000])
    first = cs.prompt_attention(q, k, v, off)
    for _ in range(3):
        assert torch.equal(first, cs.prompt_attention(q, k, v, off))
    part = cs.prompt_attention(q[:, 4:], k[:, 1:], v[:, 1:], off)
    want, mag, smag = more.prompt(q[:, 4:], k[:, 1:], v[:, 1:], [0, 1300, 2000], True, 0, 128 ** -0.5)
    close(part, want, more.prompt_bound(want, mag, smag, 1300, 128, torch.bfloat16), "part")
    close(first[:, 4:], want, more.prompt_bound(want, mag, smag, 1300, 128, torch.bfloat16), "whole")


def same(got, want):
    return bool(np.array_equal(got.cpu().numpy(), want))


# ---- codes ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,i", [(1, 1), (3, 7), (5, 16), (2, 100), (300, 129), (7, 4096), (2, 20001), (70000, 3)])
def test_quantize_rows_is_exact(dtype, m, i):
    say("case quantize", dtype, m, i)
    x = randn(gen(i), m, i, dtype=DT[dtype]) * torch.logspace(-30, 30, m, device=DEV)[:, None].to(DT[dtype])
    codes, scales = cs.quantize_rows(x)
    want, ws = more.quantize(x)
    assert codes.shape == x.shape and same(codes, want) and same(scales, ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows_of_odd_values(dtype):
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(8, 37, device=DEV)
    x[1, 3], x[2, 4], x[2, 5], x[3, :] = inf, nan, -2.0, nan
    x[4, 0], x[4, 1], x[4, 2] = -inf, 1.0, inf
    x[5], x[6, 9], x[7, 1] = torch.arange(-18, 19, device=DEV) * 0.5, 3e38, 1e-38
    x = x.to(DT[dtype])
    codes, scales = cs.quantize_rows(x)
    want, ws = more.quantize(x)
    assert same(codes, want) and same(scales, ws)


def test_quantize_rows_of_views():
    x = randn(gen(1), 6, 5, 90, dtype=torch.bfloat16)
    for t in (x, x[:, :, 3:50], x[1:, ::2], x.transpose(0, 1), x[..., ::2], x[0, 0], x[:0]):
        codes, scales = cs.quantize_rows(t)
        assert codes.shape == t.shape and scales.shape == t.shape[:-1]
        if t.numel():
            want, ws = more.quantize(t)
            assert same(codes, want) and same(scales, ws)


def check_int8(x, w, b, act, r, dtype, codes, out=None):
    wc, ws = cs.quantize_rows(w)
    if codes:
        xc, xs = cs.quantize_rows(x)
        y = cs.linear_int8(xc, wc, ws, b, act=act, residual=r, x_scale=xs, dtype=dtype, out=out)
    else:
        y = cs.linear_int8(x, wc, ws, b, act=act, residual=r, dtype=dtype, out=out)
    (xq, xsq), (wq, wsq) = more.quantize(x), more.quantize(w)
    want, bound = more.linear_int8(xq, xsq, wq, wsq, b, act, r)
    bound = bound + ref.half_ulp(dtype) * (want.abs() + bound) + 1e-37
    # What lies beyond the type's largest number rounds to infinity.
    want = torch.where(want.abs() > 1.01 * torch.finfo(dtype).max, want * math.inf, want)
    close(y, want, bound, "int8")
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,i,o", [(1, 64, 64), (1, 1, 1), (1, 4096, 130), (2, 100, 33), (7, 129, 500), (16, 2048, 16),
                                   (17, 300, 40), (40, 1000, 1003), (65, 64, 65), (129, 257, 300), (300, 2043, 257),
                                   (513, 640, 514), (1100, 130, 900)])
@pytest.mark.parametrize("codes", [False, True])
def test_int8_sizes(dtype, m, i, o, codes):
    say("case int8", dtype, m, i, o, codes, cs.describe_linear_int8(m, i, o, DT[dtype], codes))
    g = gen(m + i + o)
    x, w = randn(g, m, i, dtype=DT[dtype]), randn(g, o, i, dtype=DT[dtype]) * i ** -0.5
    check_int8(x, w, randn(g, o, dtype=DT[dtype]), "none", randn(g, m, o, dtype=DT[dtype]), DT[dtype], codes)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", list(cs.ACTIVATIONS))
@pytest.mark.parametrize("m", [3, 70, 400])
def test_int8_epilogues(dtype, act, m):
    say("case int8 epilogue", dtype, act, m)
    g, dt = gen(m), DT[dtype]
    x, w = randn(g, m, 192, dtype=dt) * 2, randn(g, 260, 192, dtype=dt) * 0.1
    for b in (None, randn(g, 260, dtype=dt)):
        for r in (None, randn(g, m, 260, dtype=dt)):
            check_int8(x, w, b, act, r, dt, True)


def test_int8_tiles_of_256_and_parts():
    """Sizes whose tiles fill the card, and few tiles over a long reduction, whose whole-number parts are joined."""
    for m, i, o, dt in ((4090, 1023, 4090, torch.bfloat16), (64, 16384, 320, torch.bfloat16),
                        (100, 9000, 200, torch.float32)):
        say("case int8", m, i, o, cs.describe_linear_int8(m, i, o, dt, True))
        g = gen(m)
        x, w = randn(g, m, i, dtype=dt), randn(g, o, i, dtype=dt) * i ** -0.5
        b = randn(g, o, dtype=dt)
        y = check_int8(x, w, b, "silu", None, dt, True)
        assert torch.equal(y, check_int8(x, w, b, "silu", None, dt, True))
    assert "256x256" in cs.describe_linear_int8(4090, 1023, 4090)
    assert "split=1 " not in cs.describe_linear_int8(64, 16384, 320)


def test_int8_largest_sums_are_exact():
    """All codes at their ends over the longest reduction: 131071 * 128 * 128 stays within 32 bits."""
    i = 131071
    for m in (2, 40):
        x = torch.full((m, i), -128, dtype=torch.int8, device=DEV)
        w = torch.full((20, i), -128, dtype=torch.int8, device=DEV)
        w[1] = 127
        one = torch.ones(m, device=DEV)
        y = cs.linear_int8(x, w, torch.ones(20, device=DEV), x_scale=one, dtype=torch.float32)
        assert float(y[0, 0]) == float(np.float32(i * 128 * 128))
        assert float(y[m - 1, 1]) == -float(np.float32(i * 128 * 127))


@pytest.mark.parametrize("m", [3, 60])
def test_int8_views_and_junk_behind_rows(m):
    """Codes in slices of wider rows: what lies behind a row, or in no row, has no influence; odd alignments."""
    g = gen(m)
    wide_x = torch.randint(-128, 128, (m, 200), generator=g, device=DEV, dtype=torch.int8)
    wide_w = torch.randint(-128, 128, (50, 208), generator=g, device=DEV, dtype=torch.int8)
    xs, ws = torch.rand(m, generator=g, device=DEV), torch.rand(50, generator=g, device=DEV) * 1e-3
    for x, w in ((wide_x[:, :100], wide_w[:, :100]), (wide_x[:, 1:100], wide_w[:, 1:100]),
                 (wide_x[:, 16:112], wide_w[:, 16:112]), (wide_x[:, 100:], wide_w[:, 108:]),
                 (wide_x[:, :190:2], wide_w[:, :190:2]), (wide_x[:, :37].contiguous(), wide_w[:, :37].contiguous()),
                 (wide_x[:, 193:], wide_w[:, 201:])):
        out = torch.full((m, 60), 9.0, device=DEV)
        cs.linear_int8(x, w, ws, x_scale=xs, dtype=torch.float32, out=out[:, 3:53])
        want, bound = more.linear_int8(*(t.cpu().numpy() for t in (x, xs, w, ws)), None, "none", None)
        close(out[:, 3:53], want, bound + 2.0 ** -24 * want.abs() + 1e-37, "view")
        assert bool((out[:, :3] == 9).all()) and bool((out[:, 53:] == 9).all())


def test_int8_scales_far_apart():
    """The product of two scales may leave fp32 where the result does not."""
    x = torch.tensor([[1e-28] * 32, [3e38] * 32, [0.0] * 32], device=DEV)
    w = torch.tensor([[1e30] * 32, [1e-30] * 32, [0.0] * 32], device=DEV)
    check_int8(x, w, None, "none", None, torch.float32, False)


def test_int8_residual_in_place_and_leading_dimensions():
    g = gen(2)
    x, w, r = (randn(g, *n, dtype=torch.bfloat16) for n in ((3, 5, 64), (48, 64), (3, 5, 48)))
    wc, ws = cs.quantize_rows(w)
    want = cs.linear_int8(x, wc, ws, residual=r)
    xc, xs = cs.quantize_rows(x)
    assert torch.equal(want, cs.linear_int8(xc, wc, ws, residual=r, x_scale=xs))
    got = r.clone()
    assert cs.linear_int8(x, wc, ws, residual=got, out=got) is got and torch.equal(got, want)
    assert cs.linear_int8(x[:0], wc, ws).shape == (0, 5, 48)


@pytest.mark.parametrize("m", [1, 2, 3, 50])
def test_int8_results_of_another_type_than_the_rows(m):
    g = gen(m)
    x, w = randn(g, m, 90), randn(g, 70, 90) * 0.1
    for a, b in ((torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)):
        check_int8(x.to(a), w, randn(g, 70, dtype=b), "relu", randn(g, m, 70, dtype=b), b, False)


def test_int8_of_one_row_without_leading_dimensions():
    g = gen(12)
    x, w = randn(g, 48, dtype=torch.bfloat16), randn(g, 33, 48, dtype=torch.bfloat16)
    wc, ws = cs.quantize_rows(w)
    xc, xs = cs.quantize_rows(x)
    want = cs.linear_int8(x[None], wc, ws)[0]
    assert xs.shape == () and torch.equal(cs.linear_int8(x, wc, ws), want)
    assert torch.equal(cs.linear_int8(xc, wc, ws, x_scale=xs), want)


@pytest.mark.parametrize("m", [1, 70])
def test_int8_weights_that_are_columns_of_a_table(m):
    """The result lies right behind the last row's codes."""
    g = gen(m)
    o, i = 96, 256
    wc, ws = cs.quantize_rows(randn(g, o, i))
    x = randn(g, m, i, dtype=torch.bfloat16)
    want = cs.linear_int8(x, wc, ws)
    held = torch.zeros(o * 2 * i + m * o * 2, dtype=torch.int8, device=DEV)
    w = held[:o * 2 * i].view(o, 2 * i)[:, :i]
    w.copy_(wc)
    at = (o - 1) * 2 * i + i
    out = held[at:at + m * o * 2].view(torch.bfloat16).view(m, o)
    assert torch.equal(cs.linear_int8(x, w, ws, out=out), want) and torch.equal(w, wc)


# ---- logits -----------------------------------------------------------------------

def check_logits(x, counts, seed, prompts=True, rep=True, pres=True, freq=True, bias=0, mask=0, history=True, out=None,
                 extra=0):
    g = gen(seed)
    n, vocab = x.shape
    h = torch.randint(-2 if extra else 0, min(vocab, 60) + extra, (sum(counts),), generator=g, device=DEV,
                      dtype=torch.int32)
    off = offsets_of(counts)
    pl = [c * (i % 4) // 4 for i, c in enumerate(counts)]
    kw = dict(repetition=0.5 + torch.rand(n, generator=g, device=DEV) if rep else None,
              presence=torch.rand(n, generator=g, device=DEV) if pres else None,
              frequency=torch.rand(n, generator=g, device=DEV) if freq else None)
    b = None if not bias else randn(g, *((vocab,) if bias == 1 else (n, vocab)))
    words = (vocab + 31) // 32
    m = None if not mask else torch.randint(-2 ** 31, 2 ** 31, (words,) if mask == 1 else (n, words), generator=g,
                                            device=DEV).to(torch.int32)
    if mask == 2:
        m[0] = 0
        m[n - 1] = -1
    if history:
        kw.update(history=h, offsets=ints(off), prompt_lengths=ints(pl) if prompts else None)
    else:
        kw = {}
    want, mag = more.logits(x, h.tolist() if history else None, off, pl if prompts else None,
                            *(kw.get(k) for k in ("repetition", "presence", "frequency")), b, m)
    y = cs.adjust_logits(x, bias=b, mask=m, out=out, **kw)
    size = torch.where(torch.isfinite(want), want.abs(), 0.0)
    bound = 6 * 2.0 ** -24 * mag + 1.01 * ref.half_ulp(x.dtype) * size + 1e-37
    close(y, want, bound, "logits")
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", [(1, 1), (1, 7), (3, 33), (2, 1000), (5, 8191), (4, 8192), (3, 8200), (2, 50021)])
@pytest.mark.parametrize("bias,mask", [(0, 0), (1, 2), (2, 1)])
def test_logits_sizes(dtype, n, vocab, bias, mask):
    say("case logits", dtype, n, vocab, bias, mask)
    x = randn(gen(vocab), n, vocab, dtype=DT[dtype]) * 3
    check_logits(x, [(37 * (i + 1)) % 150 for i in range(n)], vocab, bias=bias, mask=mask)


@pytest.mark.parametrize("prompts", [True, False])
@pytest.mark.parametrize("rep,pres,freq", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 0), (1, 1, 0)])
def test_logits_penalties_alone(prompts, rep, pres, freq):
    check_logits(randn(gen(4), 4, 500), [0, 3000, 1, 77], 5, prompts, rep, pres, freq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,seen", [(3, 700, 4100), (40, 60001, 30), (33, 70000, 30), (260, 33000, 4000)])
def test_logits_of_many_rows_and_long_histories(dtype, n, vocab, seen):
    """Every width of a workgroup; the last of these only where rows differ from the adjusted logits of one alone."""
    say("case logits", dtype, n, vocab, seen)
    x = randn(gen(n), n, vocab, dtype=DT[dtype])
    if n < 100:
        check_logits(x, [seen + i % 3 for i in range(n)], n, mask=1)
        return
    h = torch.randint(0, vocab, (n * seen,), generator=gen(1), device=DEV, dtype=torch.int32)
    off = torch.arange(n + 1, device=DEV, dtype=torch.int32) * seen
    p = [0.5 + torch.rand(n, generator=gen(2 + i), device=DEV) for i in range(3)]
    whole = cs.adjust_logits(x, h, off, None, *p)
    for b in (0, 1, 130, 259):
        one = cs.adjust_logits(x[b:b + 1], h[b * seen:(b + 1) * seen], ints([0, seen]), None, *(t[b:b + 1] for t in p))
        assert torch.equal(whole[b], one[0])


def test_logits_history_of_nothing_and_tokens_outside():
    x = randn(gen(4), 4, 50, dtype=torch.bfloat16)
    check_logits(x, [0, 0, 0, 0], 1)
    check_logits(x, [100, 0, 5, 40], 2, extra=30)
    assert torch.equal(cs.adjust_logits(x), x)
    check_logits(x, [0] * 4, 1, history=False, mask=2, bias=2)


def test_logits_odd_values_in_place_and_views():
    x = randn(gen(7), 6, 300)
    x[0, 3], x[1, 5], x[2, 7] = float("inf"), -float("inf"), float("nan")
    h, off = ints([3, 5, 7] * 6), ints([0, 3, 6, 9, 12, 15, 18])
    r, one = torch.full((6,), 1.5, device=DEV), torch.ones(6, device=DEV)
    mask = torch.full((6, 10), -1, dtype=torch.int32, device=DEV)
    mask[2, 0] = ~(1 << 7)
    kw = dict(history=h, offsets=off, repetition=r, presence=one, frequency=one, mask=mask)
    y = cs.adjust_logits(x, **kw)
    assert y[0, 3] == float("inf") and y[1, 5] == -float("inf") and y[2, 7] == -float("inf")
    same = x.clone()
    assert cs.adjust_logits(same, out=same, **kw) is same and torch.equal(same, y)
    wide = torch.full((6, 307), 4.0, device=DEV)
    wide[:, 2:302] = x
    got = cs.adjust_logits(wide[:, 2:302], out=wide[:, 2:302], **kw)
    assert torch.equal(got, y) and bool((wide[:, :2] == 4).all()) and bool((wide[:, 302:] == 4).all())
    assert torch.equal(cs.adjust_logits(x.t().contiguous().t(), **kw), y)
    assert cs.adjust_logits(x[:0]).shape == (0, 300)


# ---- streams and graphs -------------------------------------------------------------

def test_replayed_on_new_inputs_and_another_stream():
    g = gen(11)
    q, k, v = heads_of(g, 300, 4, 2, 20, torch.bfloat16)
    w, x = randn(g, 200, 100, dtype=torch.bfloat16), randn(g, 33, 100, dtype=torch.bfloat16)
    wc, ws = cs.quantize_rows(w)
    off, h, ho = ints([0, 111, 300]), ints(list(range(66))), ints(list(range(0, 68, 2)))
    one = torch.full((33,), 1.3, device=DEV)

    def calls():
        y = cs.linear_int8(x, wc, ws, act="silu")
        z = cs.adjust_logits(y, history=h, offsets=ho, repetition=one, presence=one)
        return cs.prompt_attention(q, k, v, off), y, z

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for i in range(4):
        for t in (q, x):
            t.copy_(randn(gen(50 + i), *t.shape, dtype=t.dtype))
        graph.replay()
        eager = calls()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            again = calls()
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(again, eager):
            assert torch.equal(a, b)


def test_logits_of_the_longest_history():
    """A row's tokens may be the last before the largest 32-bit number."""
    n = 2 ** 31 - 1
    history = torch.full((n,), 7, dtype=torch.int32, device=DEV)
    history[-5:] = ints([3, 900, 3, 5, 3])
    x = torch.ones(3, 1000, device=DEV)
    y = cs.adjust_logits(x, history=history, offsets=ints([0, 2, 2, 2]),
                         frequency=torch.full((3,), 0.25, device=DEV))
    want = x.clone()
    want[0, 7] = 0.5
    assert torch.equal(y, want)
    y = cs.adjust_logits(x[:1], history=history, offsets=ints([n - 5, n]), prompt_lengths=ints([1]),
                         repetition=torch.full((1,), 2.0, device=DEV), frequency=torch.full((1,), 0.25, device=DEV))
    want = x[:1].clone()
    want[0, 3], want[0, 5], want[0, 900] = 0.0, 0.25, 0.25
    assert torch.equal(y, want)


def test_two_streams_at_once():
    """Calls share nothing: two streams' results are those of one after the other."""
    g = gen(21)
    sets = []
    for n in (700, 531):
        q, k, v = heads_of(g, n, 8, 2, 60, torch.bfloat16)
        w, x = randn(g, 512, 1000, dtype=torch.bfloat16), randn(g, n, 1000, dtype=torch.bfloat16)
        sets.append((q, k, v, ints([0, n // 3, n]), x, *cs.quantize_rows(w)))

    def calls(q, k, v, off, x, wc, ws):
        y = cs.linear_int8(x, wc, ws, act="gelu")
        return cs.prompt_attention(q, k, v, off), y, cs.adjust_logits(y, mask=ints([-2 ** 31 + 5] * 16))

    want = [calls(*a) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = []
        for st, a in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(calls(*a))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for t, u in zip(a, b):
                assert torch.equal(t, u)
