"""The decoder example with weights held as codes, prompts that attend to their
own keys and values, and adjusted logits, against the same network written
plainly in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

import ref_lm as ref
import ref_lm_more as more
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_spec = importlib.util.spec_from_file_location("decoder_example", os.path.join(ROOT, "examples", "decoder.py"))
decoder = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(decoder)

SMALL = dict(layers=2, hidden=96, q_heads=6, kv_heads=2, dim=16, mlp=200, vocab=50, positions=300, pages=64,
             page_size=16)


def plain(model, tokens, positions, offsets):
    def rms(x, w):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * ref.f64(w)

    def product(x, w, b=None, act="none", residual=None):
        if not isinstance(w, tuple):
            return ref.linear(x, w, b, act, residual)[0]
        codes, scales = more.quantize(x)
        return more.linear_int8(codes, scales, w[0].cpu().numpy(), w[1].cpu().numpy(), b, act, residual)[0]

    hq, hk, dim = model.q_heads, model.kv_heads, model.dim
    x = ref.f64(model.embed)[tokens]
    n = len(tokens)
    for layer in model.layers:
        heads = product(rms(x, layer["norm"]), layer["qkv"]).view(n, -1, dim)
        cos, sin = ref.f64(model.cos), ref.f64(model.sin)
        q = ref.norm_rope(heads[:, :hq], layer["q_norm"], positions, cos, sin, 1e-6, True, False)[0]
        k = ref.norm_rope(heads[:, hq:hq + hk], layer["k_norm"], positions, cos, sin, 1e-6, True, False)[0]
        a = more.prompt(q, k, heads[:, hq + hk:], offsets, True, 0, 1 / math.sqrt(dim))[0]
        x = product(a.reshape(n, -1), layer["proj"], None, "none", x)
        h = product(rms(x, layer["mlp_norm"]), layer["up"], layer["up_bias"], "gelu_tanh")
        x = product(h, layer["down"], None, "none", x)
    return product(rms(x, model.norm), model.head)


@pytest.mark.parametrize("weights", [None, "int8"])
def test_fresh_prompts_in_fp32_against_64_bits(weights):
    """The operators are good to some 2^-18 of the hidden values here.  Without codes a chain of ten of them, each
    adding as much and none with a gain above a few, stays within 2^-12 of the largest logit.  With codes, a number so
    near the middle between two of them that 2^-18 decides gives a code's difference, 2^-7 of its row's largest, to one
    of 16 or more products: 2^-5 lies above a few such, and a wrong row, scale or mask moves logits by their own size."""
    say("case fresh prompts", weights)
    model = decoder.Decoder(weights=weights, direct=True, dtype=torch.float32, **SMALL)
    dev = model.embed.device
    new, g = [30, 1, 17], torch.Generator().manual_seed(3)
    tokens = torch.randint(0, SMALL["vocab"], (sum(new),), generator=g)
    positions, offsets = [i for n in new for i in range(n)], [0, 30, 31, 48]
    table = [[3, 0, 9, 4], [7, 1, 2, 8], [5, 6, 10, 11]]
    want = plain(model, tokens, positions, offsets)
    got = model.forward(tokens.to(dev), *(torch.tensor(v, dtype=torch.int32, device=dev)
                                          for v in (positions, table, [0, 0, 0], new, offsets)), fresh=True)
    share = 2.0 ** -12 if weights is None else 2.0 ** -5
    assert float((ref.f64(got) - want).abs().max()) <= share * float(want.abs().max())


@pytest.mark.parametrize("weights", [None, "int8"])
def test_replayed_steps_give_the_tokens_of_eager_ones(weights):
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, SMALL["vocab"], (n,), generator=g).tolist() for n in (40, 1, 23, 100)]
    found = [decoder.Decoder(weights=weights, direct=True, **SMALL).generate(prompts, 30, graph, 1.3, 0.2)[0]
             for graph in (False, True, True)]
    assert found[0].shape == (4, 30) and torch.equal(found[0], found[1]) and torch.equal(found[0], found[2])


def test_a_heavy_penalty_lets_no_token_come_twice():
    """48 tokens of a vocabulary of 50, each at most once where a generated token's logit falls by a thousand."""
    found = decoder.Decoder(direct=True, **SMALL).generate([[1, 2, 3], [4]], 48, True, 1.0, 1000.0)[0]
    for row in found.tolist():
        assert len(set(row)) == 48


def test_unknown_weights_are_refused():
    with pytest.raises(ValueError, match="unknown weights"):
        decoder.Decoder(weights="int4", **SMALL)
