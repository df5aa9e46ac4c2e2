"""Host-side checks of single properties of prompt attention, linear layers on
codes and logit adjustments, and that the GPU tests' bounds refuse what they are
there to refuse.  No GPU."""
import pytest
import torch

import paper_2410_08300_amd as cs
import ref_lm_more as more
import ref_prompt_bits as bits
from test_lm_more_host import INVALID, prompt, prompt_bytes, prompt_desc


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_bound_of_cancelling_values_tells_16_bits_of_a_weight_from_24(dtype):
    q, k, v, _, w, places = bits.cancelling(1, 64, 3, 8, 64, dtype)
    want, mag = bits.result(v, w, places, 3)
    limit = bits.bound(want, mag, dtype)
    w = w.float()
    assert bool(((bits.result(v, w.double(), places, 3)[0] - want).abs() <= limit).all())
    high = w.bfloat16().float()
    two = high.double() + (w - high).bfloat16().double()
    assert bool(((bits.result(v, two, places, 3)[0] - want).abs() > limit).any())


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -23), -2.5e38, 3.4e38])
def test_prompt_scales_beyond_their_range_are_refused(scale):
    """In powers of two they would be infinite: a score of zero times them is NaN."""
    assert prompt(prompt_desc(scale=scale)) == INVALID and prompt_bytes(prompt_desc(scale=scale))[0] == INVALID
    assert prompt_bytes(prompt_desc(scale=2.0 ** 127))[0] == prompt_bytes(prompt_desc(scale=-2.0 ** 127))[0] == 0


@pytest.mark.parametrize("dtype,seqs,tokens,rows,keys", [
    (torch.bfloat16, 14, 14 * 301, 128, 64), (torch.float32, 14, 14 * 301, 128, 32), (torch.bfloat16, 5, 1850, 64, 64),
    (torch.float32, 64, 192, 64, 64), (torch.bfloat16, 2, 850, 32, 128), (torch.float32, 2, 850, 32, 128)], ids=str)
def test_prompt_is_described_by_rows_and_keys(dtype, seqs, tokens, rows, keys):
    text = cs.describe_prompt_attention(seqs, tokens, 16, 8, 64, dtype)
    assert "rows=%d keys=%d " % (rows, keys) in text, text


@pytest.mark.parametrize("n,dim,causal,window", bits.F32_CASES)
def test_bound_of_fp32_prompts_refuses_16_bits(n, dim, causal, window):
    q, k, v = bits.f32_case(n, dim)
    want = more.prompt(q, k, v, [0, n], causal, window, dim ** -0.5)[0]
    limit = 2 * bits.far(bits.plain_f32(q, k, v, causal, window, dim ** -0.5), want)
    weights = bits.plain_f32(q, k, v, causal, window, dim ** -0.5, lambda w: bits.cut(w, 16))
    scores = bits.plain_f32(bits.cut(q, 16), bits.cut(k, 16), v, causal, window, dim ** -0.5)
    assert bool((bits.far(weights, want) > limit).all()) and bool((bits.far(scores, want) > limit).all())
