"""Host-side checks of the decoder operators at the ends of their ranges.  No GPU."""
import ctypes
import random
import re
import types

import numpy as np
import pytest
import torch

import paper_2410_08300_amd as cs
from paper_2410_08300_amd import _lib

from test_lm_host import (A, B, C, D, E, F, G, INVALID, attend, attention_desc, batch_desc, cache_desc, linear, linear_desc,
                          qk, qk_desc, read, write)


def attention_bytes(c, b, d):
    n = ctypes.c_size_t()
    return _lib.lib().convsel_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), ctypes.byref(d),
                                                        ctypes.byref(n))


@pytest.mark.parametrize("heads", [1, 2, 8, 65535])
def test_attention_rows_stay_within_what_the_kernels_count(heads):
    """Rows are counted in 32 bits, and a workgroup may look 32768 tiles of 16 past the last one."""
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


# Slices of a fused projection of two tokens' rows, 8 query heads, 2 key heads and 2 value heads of 64 in bf16.
ROW, Q, K, V = 12 * 64, A, A + 8 * 128, A + 10 * 128
FUSED = dict(q_token_stride=ROW, k_token_stride=ROW, q_out_token_stride=ROW, k_out_token_stride=ROW)


def test_rotation_refuses_outputs_over_what_else_the_call_reads_or_writes():
    d = qk_desc(**FUSED)
    far = dict(qo=F, ko=G)
    cases = [
        dict(qo=K), dict(ko=Q), dict(qo=F, ko=F), dict(qo=F, ko=F + 128), dict(qo=F, ko=F + 2 * ROW),  # over each other
        dict(qo=K - 128, ko=G), dict(qo=V, ko=G), dict(ko=Q + 7 * 128),   # over a part of the other's heads or tokens
        dict(qo=F, ko=F + 2 * ROW - 64),                                  # a tail over the next token's head
        dict(qw=F + 64), dict(kw=G), dict(qo=C), dict(ko=D + 64 * 4 * 32), dict(qo=E), dict(pos=F + 8)]
    for kw in cases:
        got = dict(q=Q, k=K)
        got.update(far)
        got.update(kw)
        assert qk(d, **got) == INVALID, kw
    # Heads that interleave, q k v q k v: the other's place one head further on.
    turns = dict(FUSED, q_heads=4, k_heads=4, q_head_stride=192, k_head_stride=192, q_out_head_stride=192,
                 k_out_head_stride=192)
    for kw in (dict(qo=A + 128, ko=G), dict(qo=A, ko=A + 64), dict(qo=A, ko=A + 384)):
        assert qk(qk_desc(**turns), q=A, k=A + 128, **kw) == INVALID, kw
    # One token: its strides are nobody's.
    one = qk_desc(tokens=1, q_token_stride=5, q_out_token_stride=1000000, k_out_token_stride=3)
    assert qk(one, q=A, k=B, qo=B + 128, ko=G) == INVALID


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="checks the no-device path; a GPU is present")
def test_rotation_takes_outputs_that_only_interleave_with_what_else_it_reads():
    d = qk_desc(**FUSED)
    ok = _lib.CONV_ERR_DEVICE  # every check of arguments passed
    for kw in (dict(qo=Q, ko=K), dict(qo=F, ko=G), dict(qo=F, ko=F + 8 * 128), dict(qo=F, ko=F + 10 * 128),
               dict(qo=Q, ko=V), dict(qo=F, ko=K)):
        assert qk(d, q=Q, k=K, **kw) == ok, kw
    turns = dict(FUSED, q_heads=4, k_heads=4, q_head_stride=192, k_head_stride=192, q_out_head_stride=192,
                 k_out_head_stride=192)
    for kw in (dict(qo=A, ko=A + 128), dict(qo=A + 256, ko=A + 128), dict(qo=F, ko=F + 256)):
        assert qk(qk_desc(**turns), q=A, k=A + 128, **kw) == ok, kw
    one = qk_desc(tokens=1, q_token_stride=5, q_out_token_stride=1000000, k_token_stride=0, k_out_token_stride=3)
    assert qk(one, q=A, k=A + 8 * 128, qo=A, ko=A + 8 * 128) == ok  # in place, whatever the strides of one token
    # Head-major: heads lie far apart, tokens one behind the other.
    major = dict(q_token_stride=64, q_head_stride=256, k_token_stride=64, k_head_stride=256, q_out_token_stride=64,
                 q_out_head_stride=256, k_out_token_stride=64, k_out_head_stride=256)
    assert qk(qk_desc(**major), q=A, k=A + 8 * 512, qo=A, ko=A + 8 * 512) == ok
    assert qk(qk_desc(k_heads=0, **FUSED), q=A, k=None, qo=A, ko=A) == ok  # no keys: their pointers are nobody's


def rows_of(base, tokens, ts, heads, hs, width):
    at = base + np.arange(tokens)[:, None, None] * ts + np.arange(heads)[None, :, None] * hs + np.arange(width)
    return set(at.ravel().tolist())


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="checks the no-device path; a GPU is present")
def test_rotation_finds_shared_values_as_sets_of_addresses_do():
    """Random small layouts: the call is refused where the output's elements and the other input's have one in common,
    or are not apart themselves, and nowhere else."""
    rng = random.Random(11)
    seen = {True: 0, False: 0}
    while min(seen.values()) < 400:
        t, hq, hk, dim = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 4), rng.choice((2, 4, 6))
        pick = (dim, dim + 2, 2 * dim, 3 * dim, hq * dim, (hq + hk) * dim, (hq + 2 * hk) * dim, t * dim, 48, 7)
        qo, k = (rng.choice(pick), rng.choice(pick)), (rng.choice(pick), rng.choice(pick))
        if rng.random() < 0.5:
            k = qo
        shift = rng.randint(-60, 60)
        out, other = rows_of(200, t, qo[0], hq, qo[1], dim), rows_of(200 + shift, t, k[0], hk, k[1], dim)
        apart = len(out) == t * hq * dim
        d = qk_desc(tokens=t, q_heads=hq, k_heads=hk, head_dim=dim, rotary_dim=0, q_token_stride=hq * dim,
                    q_head_stride=dim, q_out_token_stride=qo[0], q_out_head_stride=qo[1], k_token_stride=k[0],
                    k_head_stride=k[1], k_out_token_stride=hk * dim, k_out_head_stride=dim)
        st = qk(d, q=B, k=A + 2 * (200 + shift), qo=A + 2 * 200, ko=G)
        if not apart:
            assert st == INVALID
            continue
        shared = bool(out & other)
        # Rows that are apart as sets, but not as whole tokens or whole heads, are refused before.
        if st == INVALID and not shared:
            n0, s0, n1, s1 = t, qo[0], hq, qo[1]
            nested = (n0 == 1 or n1 == 1 or (s0 >= (n1 - 1) * s1 + dim and s1 >= dim)
                      or (s1 >= (n0 - 1) * s0 + dim and s0 >= dim))
            assert not nested, (t, hq, hk, dim, qo, k, shift)
            continue
        assert st == (INVALID if shared else _lib.CONV_ERR_DEVICE), (t, hq, hk, dim, qo, k, shift)
        seen[shared] += 1


# us by rows and in tiles, as measured with weights from memory.
FEW_ROWS = [("bf16", 1, 4096, 16384, 27.8, 38.1), ("bf16", 1, 4096, 32000, 50.7, 59.1), ("bf16", 1, 8192, 8192, 28.0, 37.2),
            ("bf16", 1, 16384, 4096, 32.3, 36.7), ("bf16", 4, 4096, 14336, 28.0, 31.6), ("bf16", 4, 4096, 16384, 29.6, 37.9),
            ("bf16", 4, 8192, 8192, 28.3, 36.2), ("bf16", 4, 11008, 4100, 29.9, 25.5), ("bf16", 16, 4096, 5120, 18.7, 14.8),
            ("bf16", 16, 5000, 5120, 24.5, 19.7), ("f32", 16, 5000, 5120, 52.7, 42.4), ("f32", 16, 11008, 4100, 85.4, 65.1),
            ("bf16", 1, 4096, 4096, 9.0, 12.8), ("bf16", 1, 14088, 541, 18.6, 12.4), ("bf16", 16, 4096, 32000, 71.8, 59.4),
            ("f32", 1, 4096, 32000, 107.5, 152.1), ("f32", 4, 14088, 541, 47.9, 25.3)]


@pytest.mark.parametrize("case", FEW_ROWS, ids=lambda c: "%s-%dx%dx%d" % c[:4])
def test_linear_of_few_rows_goes_the_faster_way(case):
    dtype, m, i, o, rows, tiles = case
    text = cs.describe_linear(m, i, o, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype])
    assert ("linear_rows_kernel" in text) == (rows < tiles), text


@pytest.mark.parametrize("prompt,singles,heads", [(4096, 127, 32), (4096, 7, 32), (512, 31, 8), (300, 600, 16), (1, 63, 8)])
def test_a_prompt_among_single_tokens_has_its_own_tiles_of_rows(prompt, singles, heads):
    """As many workgroups a key head as the prompt has tiles and the other sequences need, and less than one a sequence
    more: a plan by the average length left a prompt of 4096 tokens one of them."""
    cache = types.SimpleNamespace(_desc=ctypes.byref(cache_desc(pages=4096, kv_heads=8)), head_dim=64)
    text = cs.describe_attention(cache, 1 + singles, prompt + singles, 512, heads)
    rows, tiles = (int(re.search(r" %s=(\d+)" % n, text).group(1)) for n in ("rows", "tiles"))
    group = heads // 8
    need = -(-prompt * group // rows) + singles * -(-group // rows)
    assert need <= tiles <= need + singles + 1, text


def test_cache_reads_and_attention_refuse_outputs_over_their_batch():
    """Every workgroup reads the table, the lengths and the offsets while others write."""
    c, b, d = cache_desc(pages=4096), batch_desc(), attention_desc()
    far = F + (1 << 20)
    for at in (E, E + 28, E + 4096, E + 4100, E + 8192, E + 8196):
        assert read(c, b, k=at, v=far) == INVALID and read(c, b, k=far, v=at) == INVALID, hex(at)
        assert attend(c, b, d, y=at) == INVALID, hex(at)
        # ... and where they only end over it: 10 tokens of 2 heads (4 of queries) of 64 in bf16
        assert read(c, b, k=at - 2558, v=far) == INVALID and attend(c, b, d, y=at - 5118) == INVALID, hex(at)


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 25])
def test_rows_that_reach_further_than_64_bits_count_are_refused(n):
    """Their last byte lies 2^64 and more behind the first: no check of overlaps could count it."""
    far = 2 ** 40
    for kw in (dict(ldx=far), dict(ldy=far), dict(ldr=far, has_residual=1)):
        d = linear_desc(m=n, out_features=8, in_features=8, **dict(dict(ldx=8, ldy=8, ldr=8), **kw))
        assert linear(d, r=E if d.has_residual else None, ws=G, nws=1 << 60) == INVALID, kw
    for name in ("q_token_stride", "k_token_stride", "q_out_token_stride", "k_out_token_stride"):
        assert qk(qk_desc(tokens=n, **{name: far})) == INVALID, name
    c, b = cache_desc(pages=4096), batch_desc(seqs=1, tokens=n)
    for i in (0, 2):
        strides = [128, 64, 128, 64]
        strides[i] = far
        assert write(c, b, strides=strides) == INVALID
    one = cache_desc(pages=4096, kv_heads=1, head_dim=1)
    for name in ("q_token_stride", "y_token_stride"):
        strides = dict(dict(q_token_stride=1, q_head_stride=1, y_token_stride=1, y_head_stride=1), **{name: far})
        assert attention_bytes(one, batch_desc(seqs=1, tokens=2 ** 25), attention_desc(q_heads=1, **strides)) == INVALID
    # A stride that only one row has is nobody's.
    assert attention_bytes(one, batch_desc(seqs=1, tokens=1), attention_desc(q_heads=1, **strides)) == _lib.CONV_OK
