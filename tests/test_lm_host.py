"""Host-side checks of the decoder operators: exports, structures, refusals
before any device call, and the Python layer's own checks.  No GPU."""
import ctypes
import os
import re

import pytest
import torch

import paper_2410_08300_amd as cs
from paper_2410_08300_amd import _lib

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "convsel_lm.h")
INVALID, WORKSPACE = _lib.CONV_ERR_INVALID_ARG, _lib.CONV_ERR_WORKSPACE
A, B, C, D, E, F, G = ((i + 1) << 32 for i in range(7))  # addresses that no host check may touch


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(convsel_[a-z_0-9]*)\s*\(", text)))
    assert names == sorted(_lib.EXPORTED_LM)
    for n in names:
        assert hasattr(_lib.lib(), n), n


def test_structures_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    for c_name, cls in (("convsel_linear_desc", _lib.LinearDesc), ("convsel_qk_desc", _lib.QkDesc),
                        ("convsel_kv_cache", _lib.KvCacheDesc), ("convsel_kv_batch", _lib.KvBatchDesc),
                        ("convsel_attention_desc", _lib.AttentionDesc)):
        body = re.search(r"struct %s \{(.*?)\}" % c_name, text, flags=re.S).group(1)
        fields = []
        for line in body.split(";"):
            line = line.strip()
            if not line:
                continue
            if "*" in line:
                fields.append((line.split("*")[1].strip(), ctypes.c_void_p))
                continue
            kind, names = line.split(None, 1)
            c_type = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}[kind]
            fields += [(n.strip(), c_type) for n in names.split(",")]
        assert fields == list(cls._fields_), c_name


def test_names_of_activations_and_formats_follow_the_header():
    text = open(HEADER).read()
    for name, value in cs.ACTIVATIONS.items():
        assert re.search(r"CONVSEL_ACT_%s = %d\b" % (name.upper(), value), text), name
    for name, value in cs.FORMATS.items():
        assert re.search(r"CONVSEL_KV_%s = %d\b" % (name.upper(), value), text), name


def linear_desc(**kw):
    d = dict(m=4, in_features=64, out_features=32, ldx=64, ldr=32, ldy=32, dtype=1, act=0, has_bias=0, has_residual=0)
    d.update(kw)
    return _lib.LinearDesc(**d)


def linear(d, x=A, w=B, b=None, r=None, y=C, ws=None, nws=0):
    return _lib.lib().convsel_linear(x, w, b, r, y, ctypes.byref(d) if d else None, ws, nws, None)


@pytest.mark.parametrize("kw", [
    dict(m=-1), dict(in_features=0), dict(out_features=0), dict(m=1 << 31), dict(in_features=1 << 31),
    dict(out_features=1 << 31), dict(m=1 << 20, out_features=1 << 20), dict(dtype=2), dict(act=5), dict(act=-1),
    dict(has_bias=2), dict(has_residual=-1), dict(ldx=63), dict(ldy=31), dict(has_residual=1, ldr=31),
    dict(ldx=1 << 50)], ids=lambda k: "-".join("%s=%s" % e for e in k.items()))
def test_linear_refuses_descriptors(kw):
    d = linear_desc(**kw)
    assert linear(d, b=D if d.has_bias else None, r=E if d.has_residual else None) == INVALID
    n = ctypes.c_size_t()
    assert _lib.lib().convsel_linear_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == INVALID


def test_linear_refuses_pointers():
    d = linear_desc()
    assert linear(None) == INVALID
    assert linear(d, x=None) == INVALID and linear(d, w=None) == INVALID and linear(d, y=None) == INVALID
    assert linear(d, b=D) == INVALID and linear(d, r=D) == INVALID
    assert linear(linear_desc(has_bias=1)) == INVALID and linear(linear_desc(has_residual=1)) == INVALID
    assert linear(d, x=A + 1) == INVALID and linear(d, y=C + 1) == INVALID
    assert linear(d, y=A + 64) == INVALID and linear(d, y=B + 128) == INVALID
    assert linear(linear_desc(has_bias=1), b=C) == INVALID
    r = linear_desc(has_residual=1)
    assert linear(r, r=C + 64) == INVALID
    assert linear(linear_desc(has_residual=1, ldr=40), r=C) == INVALID  # in place, but with another stride
    assert linear(linear_desc(m=0), x=None, w=None, y=None) == _lib.CONV_OK
    n = ctypes.c_size_t()
    big = linear_desc(m=4, in_features=8192, out_features=64, ldx=8192, ldr=64, ldy=64)
    assert _lib.lib().convsel_linear_workspace_bytes(ctypes.byref(big), ctypes.byref(n)) == _lib.CONV_OK
    if n.value:
        assert linear(big, ws=D, nws=n.value - 1) == WORKSPACE and linear(big, ws=None, nws=n.value) == WORKSPACE
        assert linear(big, ws=D + 16, nws=n.value) == INVALID and linear(big, ws=C, nws=n.value) == INVALID
    assert _lib.lib().convsel_linear_workspace_bytes(ctypes.byref(d), None) == INVALID
    assert _lib.lib().convsel_linear_describe(ctypes.byref(d), None, 0) == INVALID


def qk_desc(**kw):
    d = dict(tokens=4, q_heads=8, k_heads=2, head_dim=64, rotary_dim=64, q_token_stride=512, q_head_stride=64,
             k_token_stride=128, k_head_stride=64, q_out_token_stride=512, q_out_head_stride=64,
             k_out_token_stride=128, k_out_head_stride=64, max_position=100, dtype=1, norm=1, interleaved=0, eps=1e-6)
    d.update(kw)
    return _lib.QkDesc(**d)


def qk(d, q=A, k=B, qw=None, kw=None, pos=C, cos=D, sin=E, qo=F, ko=G):
    return _lib.lib().convsel_qk_norm_rope(q, k, qw, kw, pos, cos, sin, qo, ko, ctypes.byref(d), None)


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(q_heads=-1), dict(k_heads=70000), dict(head_dim=0), dict(head_dim=1025), dict(rotary_dim=65),
    dict(rotary_dim=66), dict(rotary_dim=-2), dict(dtype=7), dict(norm=2), dict(interleaved=2), dict(eps=-1.0),
    dict(eps=float("nan")), dict(max_position=0), dict(q_token_stride=-1), dict(q_out_token_stride=511),
    dict(q_out_head_stride=63), dict(k_out_token_stride=64), dict(q_out_token_stride=0)],
    ids=lambda k: "-".join("%s=%s" % e for e in k.items()))
def test_qk_norm_rope_refuses_descriptors(kw):
    assert qk(qk_desc(**kw)) == INVALID


def test_qk_norm_rope_refuses_pointers():
    d = qk_desc()
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(cos=None), dict(sin=None), dict(qo=None), dict(ko=None),
               dict(q=A + 1), dict(pos=C + 2), dict(qw=D + 1), dict(qo=A + 64), dict(ko=B + 2)):
        assert qk(d, **kw) == INVALID, kw
    assert qk(qk_desc(q_token_stride=600), qo=A) == INVALID  # in place, but with other strides
    assert qk(qk_desc(tokens=0), q=None, k=None) == _lib.CONV_OK


def cache_desc(**kw):
    d = dict(pages=16, kv_heads=2, head_dim=64, page_size=16, format=0, k_codes=A, v_codes=B, k_scales=C, v_scales=D)
    d.update(kw)
    return _lib.KvCacheDesc(**d)


def batch_desc(**kw):
    d = dict(seqs=2, tokens=10, table_width=4, table=E, lengths=E + 4096, offsets=E + 8192)
    d.update(kw)
    return _lib.KvBatchDesc(**d)


def attention_desc(**kw):
    d = dict(q_heads=4, dtype=1, causal=1, window=0, scale=0.125, q_token_stride=256, q_head_stride=64,
             y_token_stride=256, y_head_stride=64)
    d.update(kw)
    return _lib.AttentionDesc(**d)


def write(c, b, k=F, v=F + (1 << 20), dtype=1, strides=(128, 64, 128, 64)):
    return _lib.lib().convsel_kv_write(ctypes.byref(c), ctypes.byref(b), k, v, *strides, dtype, None)


def read(c, b, k=F, v=F + (1 << 20), dtype=1):
    return _lib.lib().convsel_kv_read(ctypes.byref(c), ctypes.byref(b), k, v, dtype, None)


def attend(c, b, d, q=F, y=G, ws=F + (1 << 30), nws=1 << 28):
    return _lib.lib().convsel_attention(q, ctypes.byref(c), ctypes.byref(b), y, ctypes.byref(d), ws, nws, None)


BAD_CACHES = [dict(pages=0), dict(pages=1 << 31), dict(kv_heads=0), dict(kv_heads=40000), dict(head_dim=0),
              dict(head_dim=257), dict(page_size=8), dict(page_size=48), dict(page_size=256), dict(format=2),
              dict(k_codes=None), dict(v_codes=None), dict(k_scales=None), dict(v_scales=None), dict(k_codes=A + 8),
              dict(v_scales=D + 2)]
BAD_BATCHES = [dict(seqs=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(table_width=-1), dict(table_width=1 << 27),
               dict(table=None), dict(lengths=None), dict(offsets=None), dict(offsets=E + 2)]


@pytest.mark.parametrize("kw", BAD_CACHES, ids=lambda k: "-".join("%s=%s" % e for e in k.items()))
def test_cache_calls_refuse_caches(kw):
    c, b = cache_desc(**kw), batch_desc()
    assert write(c, b) == INVALID and read(c, b) == INVALID and attend(c, b, attention_desc(q_heads=80000)) == INVALID
    assert attend(c, b, attention_desc()) == INVALID


@pytest.mark.parametrize("kw", BAD_BATCHES, ids=lambda k: "-".join("%s=%s" % e for e in k.items()))
def test_cache_calls_refuse_batches(kw):
    c, b = cache_desc(), batch_desc(**kw)
    assert write(c, b) == INVALID and read(c, b) == INVALID and attend(c, b, attention_desc()) == INVALID


def test_cache_calls_refuse_pointers():
    c, b = cache_desc(), batch_desc()
    assert write(c, b, k=None) == INVALID and write(c, b, v=F + 1) == INVALID and write(c, b, dtype=3) == INVALID
    assert write(c, b, k=A + 64) == INVALID and write(c, b, strides=(-1, 64, 128, 64)) == INVALID
    assert read(c, b, k=None) == INVALID and read(c, b, k=F, v=F + 64) == INVALID and read(c, b, v=D) == INVALID
    assert read(c, b, dtype=9) == INVALID
    n = ctypes.c_size_t()
    L = _lib.lib()
    assert L.convsel_kv_cache_bytes(ctypes.byref(c), None) == INVALID
    assert L.convsel_kv_cache_bytes(ctypes.byref(cache_desc(head_dim=80)), ctypes.byref(n)) == _lib.CONV_OK
    assert n.value == 16 * 2 * 16 * 96
    for empty in (dict(seqs=0), dict(tokens=0)):
        e = batch_desc(table=None, lengths=None, offsets=None, **empty)
        assert write(c, e, k=None) == read(c, e, k=None) == attend(c, e, attention_desc(), q=None) == _lib.CONV_OK


@pytest.mark.parametrize("kw", [dict(q_heads=0), dict(q_heads=3), dict(q_heads=1 << 17), dict(dtype=2), dict(causal=2),
                                dict(window=-1), dict(scale=float("inf")), dict(scale=float("nan")),
                                dict(q_token_stride=-1), dict(y_token_stride=255), dict(y_head_stride=63)],
                         ids=lambda k: "-".join("%s=%s" % e for e in k.items()))
def test_attention_refuses_descriptors(kw):
    assert attend(cache_desc(), batch_desc(), attention_desc(**kw)) == INVALID


def test_attention_refuses_pointers_and_workspaces():
    c, d = cache_desc(pages=4096), attention_desc()
    b = batch_desc(seqs=1, tokens=1, table_width=2048)
    assert attend(c, b, d, q=None) == INVALID and attend(c, b, d, y=None) == INVALID and attend(c, b, d, q=F + 1) == INVALID
    assert attend(c, b, d, y=F) == INVALID and attend(c, b, d, y=A + 64) == INVALID
    n = ctypes.c_size_t()
    assert _lib.lib().convsel_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), ctypes.byref(d),
                                                        ctypes.byref(n)) == _lib.CONV_OK
    if n.value:
        assert attend(c, b, d, nws=n.value - 1) == WORKSPACE and attend(c, b, d, ws=None) == WORKSPACE
        assert attend(c, b, d, ws=F + (1 << 30) + 64) == INVALID and attend(c, b, d, ws=G) == INVALID


def test_python_layer_refuses_before_the_library():
    x, w = torch.zeros(2, 8), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU only"):
        cs.linear(x, w)
    with pytest.raises(ValueError, match="unsupported dtype"):
        cs.linear(x.double(), w.double())
    with pytest.raises(ValueError, match="unknown activation"):
        cs.describe_linear(1, 8, 8, act="swish2")
    with pytest.raises(ValueError, match="GPU only"):
        cs.qk_norm_rope(torch.zeros(1, 2, 8), torch.zeros(1, 2, 8), None, None, None)
    with pytest.raises(ValueError, match="unknown cache format"):
        cs.KVCache(4, 2, 64, fmt="int4")
    with pytest.raises(ValueError, match="GPU only"):
        cs.KVCache(4, 2, 64, device="cpu")
    with pytest.raises(cs.Conv2dError):
        cs.KVCache(4, 2, 64, page_size=24, device="cpu")


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="checks the no-device path; a GPU is present")
def test_valid_calls_without_a_device_report_it():
    ws = F + (1 << 30)
    assert linear(linear_desc(), ws=ws, nws=1 << 28) == _lib.CONV_ERR_DEVICE
    assert qk(qk_desc()) == _lib.CONV_ERR_DEVICE
    assert qk(qk_desc(), qo=A, ko=B) == _lib.CONV_ERR_DEVICE  # in place is allowed
    assert linear(linear_desc(has_residual=1), r=C, ws=ws, nws=1 << 28) == _lib.CONV_ERR_DEVICE
    assert write(cache_desc(), batch_desc()) == _lib.CONV_ERR_DEVICE
    assert read(cache_desc(), batch_desc()) == _lib.CONV_ERR_DEVICE
    assert attend(cache_desc(), batch_desc(), attention_desc()) == _lib.CONV_ERR_DEVICE
