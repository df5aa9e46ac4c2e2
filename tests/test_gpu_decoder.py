"""The decoder example, whose layers chain the decoder operators, against the
same network written plainly in 64 bits, and its replayed steps against eager ones."""
import importlib.util
import math
import os

import pytest
import torch

import ref_lm as ref
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


def plain(model, fmt, tokens, positions, table, starts, lengths, offsets, caches):
    def rms(x, w):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * ref.f64(w)

    hq, hk, dim = model.q_heads, model.kv_heads, model.dim
    x = ref.f64(model.embed)[tokens]
    n = len(tokens)
    for layer, cache in zip(model.layers, caches):
        heads = ref.linear(rms(x, layer["norm"]), layer["qkv"])[0].view(n, -1, dim)
        cos, sin = ref.f64(model.cos), ref.f64(model.sin)
        q = ref.norm_rope(heads[:, :hq], layer["q_norm"], positions, cos, sin, 1e-6, True, False)[0]
        k = ref.norm_rope(heads[:, hq:hq + hk], layer["k_norm"], positions, cos, sin, 1e-6, True, False)[0]
        cache.write(k.float(), heads[:, hq + hk:].float(), table, starts, offsets)
        a = torch.as_tensor(ref.attention(q, cache, table, lengths, offsets, True, 0, 1 / math.sqrt(dim))[0])
        x = ref.linear(a.reshape(n, -1), layer["proj"], None, "none", x)[0]
        h = ref.linear(rms(x, layer["mlp_norm"]), layer["up"], layer["up_bias"], "gelu_tanh")[0]
        x = ref.linear(h, layer["down"], None, "none", x)[0]
    return ref.linear(rms(x, model.norm), model.head)[0]


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_decoder_in_fp32_against_64_bits(fmt):
    """Prompts, then two steps.  The operators are good to some 2^-18 here; beyond that, a key or value so near the
    middle between two codes that 2^-18 decides gives one code's difference, 2^-7 of it in int8 and 2^-4 in fp8, to one
    of 16 products of a score, or to one weighted value.  Hidden values are of order 1 (weights have unit gain) and the
    residual path adds them: 2^-5 and 2^-3 of the largest logit lie above a few such codes, and a wrong row, head,
    position, mask or page moves logits by their own size."""
    say("case decoder", fmt)
    model = decoder.Decoder(fmt=fmt, dtype=torch.float32, **SMALL)
    dev = model.embed.device
    table = [[3, 0, 9, 4], [7, 1, 2, 8], [5, 6, 10, 11]]
    caches = [ref.Cache(SMALL["pages"], SMALL["kv_heads"], SMALL["dim"], SMALL["page_size"], fmt) for _ in model.layers]
    g = torch.Generator().manual_seed(3)
    held = [0, 0, 0]
    for new in ([30, 1, 17], [1, 1, 1], [1, 1, 1]):
        tokens = torch.randint(0, SMALL["vocab"], (sum(new),), generator=g)
        positions = [h + i for h, n in zip(held, new) for i in range(n)]
        offsets = [0, new[0], new[0] + new[1], sum(new)]
        lengths = [h + n for h, n in zip(held, new)]
        want = plain(model, fmt, tokens, positions, table, held, lengths, offsets, caches)
        got = model.forward(tokens.to(dev), *(torch.tensor(v, dtype=torch.int32, device=dev)
                                              for v in (positions, table, held, lengths, offsets)))
        share = 2.0 ** -5 if fmt == "int8" else 2.0 ** -3
        assert float((ref.f64(got) - want).abs().max()) <= share * float(want.abs().max())
        held = lengths


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_replayed_steps_give_the_tokens_of_eager_ones(fmt):
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, SMALL["vocab"], (n,), generator=g).tolist() for n in (40, 1, 23, 100)]
    found = [decoder.Decoder(fmt=fmt, **SMALL).generate(prompts, 40, graph=graph)[0] for graph in (False, True, True)]
    assert found[0].shape == (4, 40) and torch.equal(found[0], found[1]) and torch.equal(found[0], found[2])


def test_sequences_do_not_touch_each_other():
    """Every sequence's tokens are those that the same place gets beside other sequences."""
    g = torch.Generator().manual_seed(5)
    a, b, c = ([torch.randint(0, SMALL["vocab"], (n,), generator=g).tolist() for n in (33, 20, 64)])
    first = decoder.Decoder(**SMALL).generate([a, b, c], 20)[0]
    turned = decoder.Decoder(**SMALL).generate([c, a, b], 20)[0]
    assert torch.equal(first, turned[[1, 2, 0]])


def test_generate_refuses_what_does_not_fit():
    with pytest.raises(ValueError, match="too small"):
        decoder.Decoder(**SMALL).generate([[1] * 290], 20)
