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
