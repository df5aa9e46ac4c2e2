"""Host-side checks of the decoder operators at the ends of their ranges.  No GPU."""
import ctypes

import pytest

from paper_2410_08300_amd import _lib

from test_lm_host import INVALID, attention_desc, batch_desc, cache_desc


def attention_bytes(c, b, d):
    n = ctypes.c_size_t()
    return _lib.lib().convsel_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), ctypes.byref(d),
                                                        ctypes.byref(n))


@pytest.mark.parametrize("heads", [1, 2, 8, 65535])
def test_attention_rows_stay_within_what_the_kernels_count(heads):
    """A workgroup of 16 rows goes on by up to 32768 tiles of them in 32 bits: past the last row that has to stay below
    2^31."""
    d = attention_desc(q_heads=heads, q_token_stride=heads, q_head_stride=1, y_token_stride=heads, y_head_stride=1)
    c = cache_desc(kv_heads=1, head_dim=1)
    most = (2 ** 31 - 2 ** 20) // heads
    assert most * heads + 32768 * 16 < 2 ** 31
    assert attention_bytes(c, batch_desc(seqs=1, tokens=most), d) == _lib.CONV_OK
    for tokens in (most + 1, (2 ** 31 - 1) // heads):
        assert attention_bytes(c, batch_desc(seqs=1, tokens=tokens), d) == INVALID
