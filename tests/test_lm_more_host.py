"""Host-side checks of prompt attention, linear layers on codes and logit
adjustments: structures, refusals before any device call, and the Python layer's
own checks.  No GPU."""
import ctypes
import os
import re

import pytest
import torch

import paper_2410_08300_amd as cs
from paper_2410_08300_amd import _lib

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "convsel_lm.h")
INVALID, WORKSPACE = _lib.CONV_ERR_INVALID_ARG, _lib.CONV_ERR_WORKSPACE
A, B, C, D, E, F, G, H, I, J = ((i + 1) << 32 for i in range(10))  # addresses that no host check may touch


def ident(kw):
    return "-".join("%s=%s" % e for e in kw.items())


def test_structures_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    for c_name, cls in (("convsel_prompt_desc", _lib.PromptDesc), ("convsel_quantize_desc", _lib.QuantizeDesc),
                        ("convsel_linear_int8_desc", _lib.LinearInt8Desc), ("convsel_logits_desc", _lib.LogitsDesc)):
        body = re.search(r"struct %s \{(.*?)\}" % c_name, text, flags=re.S).group(1)
        fields = []
        for line in body.split(";"):
            if line.strip():
                kind, names = line.strip().split(None, 1)
                c_type = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}[kind]
                fields += [(n.strip(), c_type) for n in names.split(",")]
        assert fields == list(cls._fields_), c_name


# ---- prompts --------------------------------------------------------------------

def prompt_desc(**kw):
    d = dict(seqs=2, tokens=10, q_heads=4, kv_heads=2, head_dim=64, dtype=1, causal=1, window=0, scale=1.0)
    for t, h in (("q", 4), ("k", 2), ("v", 2), ("y", 4)):
        d[t + "_token_stride"], d[t + "_head_stride"] = h * 64, 64
    d.update(kw)
    return _lib.PromptDesc(**d)


def prompt(d, q=A, k=B, v=C, off=D, y=E, ws=None, n=0):
    return _lib.lib().convsel_prompt_attention(q, k, v, off, y, ctypes.byref(d) if d else None, ws, n, None)


def prompt_bytes(d, q=A, k=B, v=C):
    n = ctypes.c_size_t()
    st = _lib.lib().convsel_prompt_attention_workspace_bytes(q, k, v, ctypes.byref(d), ctypes.byref(n))
    return st, n.value


@pytest.mark.parametrize("kw", [
    dict(seqs=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(seqs=1 << 31), dict(q_heads=0), dict(kv_heads=0),
    dict(q_heads=5), dict(head_dim=0), dict(head_dim=257), dict(dtype=2), dict(causal=2), dict(window=-1),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(tokens=1 << 30), dict(q_token_stride=-1),
    dict(k_head_stride=1 << 50), dict(v_token_stride=1 << 45), dict(y_head_stride=-4)], ids=ident)
def test_prompt_refuses_descriptors(kw):
    d = prompt_desc(**kw)
    assert prompt(d) == INVALID and prompt_bytes(d)[0] == INVALID


def test_prompt_refuses_pointers_and_overlaps():
    d = prompt_desc()
    assert prompt(None) == INVALID
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(off=None), dict(y=None), dict(q=A + 1), dict(k=B + 1),
               dict(v=C + 1), dict(y=E + 1), dict(off=D + 2)):
        assert prompt(d, **kw) == INVALID, kw
    # y over an input, the offsets, or its own rows.
    for kw in (dict(y=A), dict(y=A + 4 * 128), dict(y=B), dict(y=C + 128), dict(off=E + 64)):
        assert prompt(d, **kw) == INVALID, kw
    for kw in (dict(y_head_stride=63), dict(y_token_stride=255), dict(y_token_stride=0), dict(y_head_stride=0)):
        assert prompt(prompt_desc(**kw)) == INVALID, kw


def test_prompt_workspace_follows_alignment():
    assert prompt_bytes(prompt_desc()) == (0, 0)
    rows = 10 * 2 * 64 * 2
    assert prompt_bytes(prompt_desc(), k=B + 2) == (0, (rows + 255) // 256 * 256)
    assert prompt_bytes(prompt_desc(), q=A + 8)[1] == (10 * 4 * 128 + 255) // 256 * 256
    st, n = prompt_bytes(prompt_desc(head_dim=60, k_token_stride=121))
    assert st == 0 and n == (10 * 4 * 128 + 255) // 256 * 256 + 2 * ((rows + 255) // 256 * 256)
    d = prompt_desc(head_dim=60)
    assert prompt(d) == WORKSPACE and prompt(d, ws=F, n=n - 1) == WORKSPACE and prompt(d, ws=F + 8, n=n) == INVALID
    assert prompt(d, ws=A, n=n) == INVALID and prompt(d, ws=E, n=n) == INVALID and prompt(d, ws=D - 256, n=n) == INVALID


def test_prompt_rows_far_apart_are_copied():
    """A tile of 128 keys is addressed in 32 bits."""
    near, far = (1 << 31) // 128 // 2 - 256, (1 << 31) // 128 // 2
    assert prompt_bytes(prompt_desc(k_token_stride=near, v_token_stride=near)) == (0, 0)
    assert prompt_bytes(prompt_desc(k_token_stride=far))[1] == (10 * 2 * 128 + 255) // 256 * 256
    assert prompt_bytes(prompt_desc(dtype=0, v_token_stride=far // 2))[1] == 10 * 2 * 256


def test_prompt_over_nothing_is_a_no_op():
    assert prompt(prompt_desc(tokens=0), q=None, y=None) == 0 and prompt(prompt_desc(seqs=0), q=None) == 0
    assert prompt_bytes(prompt_desc(tokens=0, head_dim=3)) == (0, 0)


def test_prompt_python_refusals():
    q, k = torch.zeros(4, 4, 8), torch.zeros(4, 2, 8)
    off = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU only"):
        cs.prompt_attention(q, k, k, off)
    with pytest.raises(ValueError, match="unsupported dtype"):
        cs.prompt_attention(q.half(), k.half(), k.half(), off)
    assert "rows=" in cs.describe_prompt_attention(3, 100, 8, 2, 64)
    assert "prompt_pack_kernel" in cs.describe_prompt_attention(3, 100, 8, 2, 63)


# ---- codes ------------------------------------------------------------------------

def quantize(x=A, c=B, s=C, **kw):
    d = dict(m=4, in_features=50, ldx=50, ldc=64, dtype=1)
    d.update(kw)
    return _lib.lib().convsel_quantize_rows(x, c, s, ctypes.byref(_lib.QuantizeDesc(**d)), None)


@pytest.mark.parametrize("kw", [
    dict(m=-1), dict(m=1 << 31), dict(in_features=0), dict(in_features=1 << 31), dict(ldx=49), dict(ldc=49),
    dict(dtype=2), dict(dtype=-1), dict(ldx=1 << 50), dict(ldc=1 << 50), dict(x=None), dict(c=None), dict(s=None),
    dict(x=A + 1), dict(s=C + 2), dict(c=A), dict(s=A + 40), dict(s=B + 252), dict(c=A - 255)], ids=ident)
def test_quantize_refuses(kw):
    assert quantize(**kw) == INVALID


def int8_desc(**kw):
    d = dict(m=4, in_features=64, out_features=32, ldx=64, ldw=64, ldr=32, ldy=32, x_dtype=-1, dtype=1, act=0,
             has_bias=0, has_residual=0)
    d.update(kw)
    return _lib.LinearInt8Desc(**d)


def int8(d, x=A, xs=B, w=C, ws=D, b=None, r=None, y=E, work=None, n=0):
    return _lib.lib().convsel_linear_int8(x, xs, w, ws, b, r, y, ctypes.byref(d) if d else None, work, n, None)


def int8_bytes(d, x=A, w=C):
    n = ctypes.c_size_t()
    st = _lib.lib().convsel_linear_int8_workspace_bytes(x, w, ctypes.byref(d), ctypes.byref(n))
    return st, n.value


@pytest.mark.parametrize("kw", [
    dict(m=-1), dict(m=1 << 31), dict(in_features=0), dict(in_features=1 << 17, ldx=1 << 17, ldw=1 << 17),
    dict(out_features=0), dict(out_features=1 << 26), dict(m=1 << 20, out_features=1 << 20), dict(ldx=63), dict(ldw=63),
    dict(ldy=31), dict(has_residual=1, ldr=31), dict(x_dtype=2), dict(x_dtype=-2), dict(dtype=-1), dict(dtype=2),
    dict(act=5), dict(act=-1), dict(has_bias=2), dict(has_residual=-1), dict(ldx=1 << 50), dict(ldw=1 << 50)],
    ids=ident)
def test_int8_refuses_descriptors(kw):
    d = int8_desc(**kw)
    assert int8(d, b=F if d.has_bias else None, r=G if d.has_residual else None) == INVALID
    assert int8_bytes(d)[0] == INVALID


def test_int8_refuses_pointers_and_overlaps():
    d = int8_desc()
    assert int8(None) == INVALID
    for kw in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(y=None), dict(b=F), dict(r=G),
               dict(xs=B + 2), dict(ws=D + 1), dict(y=E + 1)):
        assert int8(d, **kw) == INVALID, kw
    for kw in (dict(y=A), dict(y=A + 254), dict(y=B + 8), dict(y=C), dict(y=D + 64), dict(y=D - 200)):
        assert int8(d, **kw) == INVALID, kw
    both = int8_desc(has_bias=1, has_residual=1)
    assert int8(both, b=E + 4, r=G) == INVALID and int8(both, b=F, r=E + 64) == INVALID
    assert int8(int8_desc(has_residual=1, ldr=40), r=E) == INVALID  # the same address with another stride
    # The residual's own place is no excuse for another operand's.
    assert int8(int8_desc(has_residual=1, x_dtype=1), x=E, xs=None, r=E, work=H, n=1 << 20) == INVALID
    # Numbers bring no scales.
    assert int8(int8_desc(x_dtype=1), work=H, n=1 << 20) == INVALID


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run on these addresses")
def test_int8_weights_end_with_their_last_row():
    """Rows of w may be columns of a wider table: what lies right behind the last one's units is not w's."""
    d, end = int8_desc(ldw=128), C + 31 * 128 + 64
    assert int8(d, y=end - 2) == INVALID and int8(d, y=end) == _lib.CONV_ERR_DEVICE
    d, end = int8_desc(in_features=60, ldx=64, ldw=128), C + 31 * 128 + 64
    work = dict(work=H, n=1 << 12)
    assert int8(d, y=end - 2, **work) == INVALID and int8(d, y=end, **work) == _lib.CONV_ERR_DEVICE


def test_int8_workspace():
    assert int8_bytes(int8_desc()) == (0, 0)
    st, n = int8_bytes(int8_desc(x_dtype=1))
    assert st == 0 and n % 256 == 0
    d = int8_desc(x_dtype=1, m=40)
    st, n = int8_bytes(d)
    assert st == 0 and n >= 40 * 64 + 40 * 4
    assert int8(d, xs=None) == WORKSPACE and int8(d, xs=None, work=H, n=n - 1) == WORKSPACE
    assert int8(d, xs=None, work=H + 16, n=n) == INVALID
    for kw in (dict(work=A), dict(work=C), dict(work=E), dict(work=D)):
        assert int8(d, xs=None, n=n, **kw) == INVALID, kw
    # Weights that do not lie in whole units are copied.
    assert int8_bytes(int8_desc(), w=C + 1)[1] >= 32 * 64 and int8_bytes(int8_desc(ldw=65))[1] >= 32 * 64
    assert int8_bytes(int8_desc(m=0, x_dtype=1)) == (0, 0) and int8(int8_desc(m=0), x=None) == 0


def test_int8_python_refusals():
    x, w, s = torch.zeros(3, 8), torch.zeros(4, 8, dtype=torch.int8), torch.ones(4)
    with pytest.raises(ValueError, match="GPU only"):
        cs.linear_int8(x, w, s)
    with pytest.raises(ValueError, match="GPU only"):
        cs.quantize_rows(x)
    with pytest.raises(ValueError, match="unsupported dtype"):
        cs.quantize_rows(x.half())
    assert "linear_int8" in cs.describe_linear_int8(1, 4096, 4096)


# ---- logits -----------------------------------------------------------------------

def logits(x=A, h=B, off=C, pl=D, rep=E, pres=F, freq=G, bias=H, mask=I, y=J, **kw):
    d = dict(rows=4, vocab=100, tokens=50, ldx=100, ldy=100, ldbias=100, ldmask=4, dtype=1)
    d.update(kw)
    return _lib.lib().convsel_adjust_logits(x, h, off, pl, rep, pres, freq, bias, mask, y,
                                            ctypes.byref(_lib.LogitsDesc(**d)), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(tokens=-1), dict(tokens=1 << 31),
    dict(ldx=99), dict(ldy=99), dict(ldbias=99), dict(ldmask=3), dict(dtype=2), dict(ldx=1 << 50), dict(ldmask=1 << 50),
    dict(x=None), dict(y=None), dict(h=None), dict(off=None), dict(h=None, off=None), dict(x=A + 1), dict(y=J + 1),
    dict(h=B + 2), dict(mask=I + 1), dict(bias=H + 2), dict(pl=D + 1), dict(y=A + 2), dict(y=A, ldx=104), dict(y=B),
    dict(y=C), dict(y=D), dict(y=E), dict(y=F + 12), dict(y=G), dict(y=H + 400), dict(y=I)], ids=ident)
def test_logits_refuse(kw):
    assert logits(**kw) == INVALID


def test_logits_over_no_rows_are_a_no_op():
    assert logits(rows=0, x=None, y=None) == 0


def test_logits_python_refusals():
    with pytest.raises(ValueError, match="GPU only"):
        cs.adjust_logits(torch.zeros(2, 5))
    with pytest.raises(ValueError, match="unsupported dtype"):
        cs.adjust_logits(torch.zeros(2, 5, dtype=torch.float64))
