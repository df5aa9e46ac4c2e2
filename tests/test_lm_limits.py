"""Host-side checks of the decoder operators at the ends of their ranges.  No GPU."""
import ctypes
import re
import types

import pytest
import torch

import paper_2410_08300_amd as cs
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


def test_a_window_of_any_size_is_the_window_asked_for():
    """2^32 + 8 is no window of eight tokens."""
    cache = types.SimpleNamespace(_desc=ctypes.byref(cache_desc(pages=4096)), head_dim=64)

    def text(window):
        return cs.describe_attention(cache, 1, 64, 4096, 4, window=window)

    assert text(8) != text(0)  # the plan shows it
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 8, 2 ** 63 - 1, 2 ** 70):
        assert text(window) == text(0)
    for window in (-1, -2 ** 32 + 8):
        with pytest.raises((ValueError, cs.Conv2dError)):
            text(window)


@pytest.mark.parametrize("kw", [dict(kv_heads=2 ** 32 + 2), dict(head_dim=2 ** 32 + 64), dict(page_size=2 ** 32 + 16)],
                         ids=lambda k: next(iter(k)))
def test_cache_sizes_that_leave_their_fields_are_refused(kw):
    sizes = dict(pages=4, kv_heads=2, head_dim=64, page_size=16, device="cpu")
    sizes.update(kw)
    with pytest.raises(ValueError, match=next(iter(kw))):
        cs.KVCache(**sizes)


@pytest.mark.parametrize("cls", [_lib.LinearDesc, _lib.QkDesc, _lib.KvCacheDesc, _lib.AttentionDesc])
def test_structures_refuse_numbers_that_leave_their_fields(cls):
    for i, (name, kind) in enumerate(cls._fields_):
        if kind not in (ctypes.c_int32, ctypes.c_int64):
            continue
        bits = 8 * ctypes.sizeof(kind)
        for value in (2 ** (bits - 1), 2 ** bits + 1, -2 ** (bits - 1) - 1):
            with pytest.raises(ValueError, match=name):
                cls(**{name: value})
            with pytest.raises(ValueError, match=name):
                cls(*([0] * i + [value]))
        for value in (2 ** (bits - 1) - 1, -2 ** (bits - 1)):
            assert getattr(cls(**{name: value}), name) == value


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("outputs", [1, 8, 16, 17, 64, 65])
def test_linear_of_very_many_rows_fits_a_launch(outputs, dtype):
    """A launch holds 2^32 threads: tiles of 256 threads, their grid rounded up to 8 of them, stay below that."""
    most = min(2 ** 31 - 1, 2 ** 35 // outputs)
    for m in (2 ** 30 - 64, 2 ** 30, 2 ** 30 + 1, most):
        if m > most:
            continue
        text = cs.describe_linear(m, 8, outputs, dtype)
        side = int(re.search(r" tile=(\d+)x", text).group(1))
        tiles = -(-m // side) * -(-outputs // side)
        assert "tiles" in text and (tiles + 7) // 8 * 8 * 256 < 2 ** 32, text
