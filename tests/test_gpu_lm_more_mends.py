"""GPU checks of single properties of prompt attention, linear layers on codes and
logit adjustments, each at the calls where it can be lost."""
import pytest
import torch

import ref_prompt_bits as bits
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2410_08300_amd as cs  # noqa: E402
from test_gpu_lm_more import DEV, DT, close, ints  # noqa: E402


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
