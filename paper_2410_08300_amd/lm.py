"""Decoder-layer operators: torch-facing calls into include/convsel_lm.h.

``linear`` (a product with bias, activation and residual in its epilogue),
``qk_norm_rope`` (norm and position rotation of query and key heads),
``KVCache`` (a paged key/value cache held in 8 bits) and ``cached_attention``
(attention over it); ``prompt_attention`` (packed prompts over their own keys and
values), ``quantize_rows`` and ``linear_int8`` (layers whose weights are held in 8
bits) and ``adjust_logits`` (penalties, biases and masks before a token is chosen).
All are forward only.  As with ``conv2d``, PyTorch supplies device memory and the
current stream, the work runs in the HIP library, and there is no CPU path.
Calls are asynchronous, and like every PyTorch operation they take tensors of
another stream only after the caller has made the current one wait for it.
"""
import ctypes
import functools
import math

import torch

from . import _lib

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
FORMATS = {"int8": 0, "fp8": 1}


def _dtype_of(what, first, *others):
    dt, dev = first.dtype, first.device
    code = _DTYPES.get(dt)
    if code is None:
        raise ValueError("%s: unsupported dtype %s (float32 or bfloat16)" % (what, dt))
    if not first.is_cuda:
        raise ValueError("%s runs on the GPU only: move its tensors to a HIP device" % what)
    for t in others:
        if t is not None and (t.dtype is not dt or t.device != dev):
            raise ValueError("%s: tensors must share one dtype and one HIP device" % what)
    return code


def _raise(st, what):
    if st:
        raise _lib.Conv2dError(st, what)


def _run(what, function, device, *args):
    """The library call on PyTorch's current stream of ``device``."""
    index = device.index
    if index == torch._C._cuda_getDevice():
        st = function(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(device):
            st = function(*args, torch._C._cuda_getCurrentRawStream(index))
    if st:
        raise _lib.Conv2dError(st, what)


# ---- linear -------------------------------------------------------------------

def _rows(t):
    """t as a matrix of rows with a dense last dimension (a view where it can
    be one), and its row stride."""
    if t.dim() == 2 and t.is_contiguous():
        return t, t.shape[1]
    m = t.reshape(-1, t.shape[-1])
    if m.stride(1) != 1 and m.shape[1] > 1 or m.stride(0) < m.shape[1] and m.shape[0] > 1:
        m = m.contiguous()
    return m, (m.stride(0) if m.shape[0] > 1 else m.shape[1])


def _linear_desc(m, i, o, ldx, ldr, ldy, dtype, act, bias, residual):
    if act not in ACTIVATIONS:
        raise ValueError("unknown activation %r (one of %s)" % (act, ", ".join(ACTIVATIONS)))
    return _lib.LinearDesc(m, i, o, ldx, ldr, ldy, dtype, ACTIVATIONS[act], bias, residual)


@functools.lru_cache(maxsize=1024)
def _linear_plan(*sizes):
    """(descriptor by reference, workspace bytes) of a call of these sizes."""
    d = ctypes.byref(_linear_desc(*sizes))
    n = ctypes.c_size_t()
    _raise(_lib.lib().convsel_linear_workspace_bytes(d, ctypes.byref(n)), "linear")
    return d, n.value


def linear(x, w, b=None, act="none", residual=None, out=None):
    """``act(x @ w.T + b) + residual`` over the last dimension of ``x``.

    ``w`` is [out_features][in_features]; ``act`` is "none", "relu", "gelu"
    (erf), "gelu_tanh" or "silu".  The sum, the activation and the residual add
    are fp32 and rounded once.  ``out`` may be ``residual`` itself.  Rows of
    ``x``, ``residual`` and ``out`` may be strided.
    """
    dt = _dtype_of("linear", x, w, b, residual, out)
    if x.dim() < 1 or w.dim() != 2 or x.shape[-1] != w.shape[1]:
        raise ValueError("linear: input features of x %s and weight %s differ" % (tuple(x.shape), tuple(w.shape)))
    o, i = w.shape
    if b is not None and tuple(b.shape) != (o,):
        raise ValueError("linear: bias must hold %d values" % o)
    shape = x.shape[:-1] + (o,)
    if residual is not None and residual.shape != shape:
        raise ValueError("linear: residual must have shape %s" % (tuple(shape),))
    if out is None:
        out = x.new_empty(shape)
    elif out.shape != shape:
        raise ValueError("linear: out must have shape %s" % (tuple(shape),))
    if i == 0 or o == 0:
        raise ValueError("linear: empty weight")
    if out.numel() == 0:
        return out
    x2, ldx = _rows(x)
    y2, ldy = _rows(out)
    if y2.data_ptr() != out.data_ptr():
        raise ValueError("linear: out must be a view of rows with a dense last dimension")
    r2, ldr = (None, 0) if residual is None else _rows(residual)
    w = w.contiguous()
    b = None if b is None else b.contiguous()
    if x2.shape[0] > 16:
        # The library's tiles read operands that start on 16 bytes; a view that does not is copied first.
        x2, ldx = (x2, ldx) if x2.data_ptr() % 16 == 0 else (x2.clone(memory_format=torch.contiguous_format), i)
        w = w if w.data_ptr() % 16 == 0 else w.clone()
    d, n = _linear_plan(x2.shape[0], i, o, ldx, ldr, ldy, dt, act, b is not None, r2 is not None)
    ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
    _run("linear", _lib.lib().convsel_linear, x.device, x2.data_ptr(), w.data_ptr(), None if b is None else b.data_ptr(),
         None if r2 is None else r2.data_ptr(), y2.data_ptr(), d, None if ws is None else ws.data_ptr(), n)
    return out


def describe_linear(m, in_features, out_features, dtype=torch.bfloat16, act="none", bias=False, residual=False):
    """How the library runs this linear layer on dense rows, as one line."""
    d = _linear_desc(m, in_features, out_features, in_features, out_features, out_features, _DTYPES[dtype], act, bias,
                     residual)
    buf = ctypes.create_string_buffer(512)
    _raise(_lib.lib().convsel_linear_describe(ctypes.byref(d), buf, len(buf)), "linear")
    return buf.value.decode()


# ---- norm and rotation ----------------------------------------------------------

def _heads(t, what):
    """t as [tokens][heads][dim] with a dense last dimension."""
    if t.dim() != 3:
        raise ValueError("%s: expected [tokens][heads][dim], got shape %s" % (what, tuple(t.shape)))
    return t if t.stride(2) == 1 or t.shape[2] == 1 else t.contiguous()


def _ints(t, n, what, device):
    if t.dtype is not torch.int32 or t.shape != n or t.device != device:
        raise ValueError("%s must be an int32 tensor of shape %s on %s" % (what, tuple(n), device))
    return t if t.is_contiguous() else t.contiguous()


@functools.lru_cache(maxsize=1024)
def _qk_plan(*sizes):
    return ctypes.byref(_lib.QkDesc(*sizes))


def qk_norm_rope(q, k, positions, cos, sin, q_weight=None, k_weight=None, eps=1e-6, norm="rms", interleaved=False,
                 q_out=None, k_out=None):
    """Norm of every head of ``q`` and ``k`` ([tokens][heads][dim], e.g. views
    of one fused projection), then the position rotation, in one pass:
    (q_out, k_out).

    ``norm`` is "rms" (x / sqrt(mean x^2 + eps) * weight) or "none" (x * weight).  ``cos``
    and ``sin`` are fp32 tables [positions][R/2], ``positions`` an int32 row of
    them per token; the first R values of a head turn, as pairs (i, i + R/2) or
    with ``interleaved`` (2i, 2i + 1).  ``cos=None`` turns nothing.  Outputs may
    be the inputs themselves.  A token whose position the tables lack is NaN.
    """
    dt = _dtype_of("qk_norm_rope", q, k, q_weight, k_weight, q_out, k_out)
    q, k = _heads(q, "qk_norm_rope"), _heads(k, "qk_norm_rope")
    (t, hq, dim), (tk, hk, dim_k), dev = q.shape, k.shape, q.device
    if tk != t or dim_k != dim:
        raise ValueError("qk_norm_rope: q %s and k %s differ in tokens or width" % (tuple(q.shape), tuple(k.shape)))
    if norm not in ("rms", "none"):
        raise ValueError("unknown norm %r (rms or none)" % (norm,))
    for wt in (q_weight, k_weight):
        if wt is not None and wt.shape != (dim,):
            raise ValueError("qk_norm_rope: a weight must hold %d values" % dim)
    if (cos is None) != (sin is None):
        raise ValueError("qk_norm_rope: cos and sin come together")
    rotary = rows = 0
    if cos is not None:
        if (cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32
                or cos.device != dev or sin.device != dev):
            raise ValueError("qk_norm_rope: cos and sin must be float32 tables of one shape on %s" % dev)
        rows, rotary = cos.shape
        rotary *= 2
        if rotary > dim:
            raise ValueError("qk_norm_rope: tables rotate %d of %d values" % (rotary, dim))
        cos, sin = cos.contiguous(), sin.contiguous()
        positions = _ints(positions, (t,), "positions", dev)
    q_weight = None if q_weight is None else q_weight.contiguous()
    k_weight = None if k_weight is None else k_weight.contiguous()
    for o, ref in ((q_out, q), (k_out, k)):
        if o is not None and (o.shape != ref.shape or (o.stride(2) != 1 and dim > 1)):
            raise ValueError("qk_norm_rope: an output must have its input's shape and a dense last dimension")
    q_out = q.new_empty((t, hq, dim)) if q_out is None else q_out
    k_out = q.new_empty((t, hk, dim)) if k_out is None else k_out
    if dim == 0:
        raise ValueError("qk_norm_rope: empty heads")
    qs, ks, qo, ko = q.stride(), k.stride(), q_out.stride(), k_out.stride()
    d = _qk_plan(t, hq, hk, dim, rotary, qs[0], qs[1], ks[0], ks[1], qo[0], qo[1], ko[0], ko[1], rows, dt,
                 1 if norm == "rms" else 0, bool(interleaved), eps)
    _run("qk_norm_rope", _lib.lib().convsel_qk_norm_rope, dev, q.data_ptr(), k.data_ptr(),
         None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
         positions.data_ptr() if rotary else None, cos.data_ptr() if rotary else None,
         sin.data_ptr() if rotary else None, q_out.data_ptr(), k_out.data_ptr(), d)
    return q_out, k_out


# ---- cache ----------------------------------------------------------------------

class _Buffer:
    """A tensor whose address the library was given: it takes new values in place, and no other tensor in its place."""

    def __set_name__(self, owner, name):
        self.name = name

    def __get__(self, obj, owner=None):
        return self if obj is None else obj.__dict__[self.name]

    def __set__(self, obj, value):
        if obj.__dict__.setdefault(self.name, value) is not value:
            raise AttributeError("KVCache.%s cannot be replaced: copy new values into it" % self.name)


class KVCache:
    """A paged key/value cache held in 8 bits: ``pages`` pages of ``page_size``
    (16, 32, 64 or 128) tokens of ``kv_heads`` heads of ``head_dim`` (up to
    256) values, with one fp32 scale per page and head for the keys and one for
    the values.  ``fmt`` is "int8" or "fp8" (e4m3).

    Which pages a sequence holds is the caller's block table, an int32 tensor
    [sequences][pages of a sequence]; an entry outside the cache (-1) is no
    page.  ``offsets`` (int32, [sequences + 1]) divides a call's packed tokens
    among the sequences.  include/convsel_lm.h has the layout of ``k_codes``,
    ``v_codes``, ``k_scales`` and ``v_scales``, and what a write does to the
    scale of a page that fills up; they take new values in place.
    """

    k_codes, v_codes, k_scales, v_scales = _Buffer(), _Buffer(), _Buffer(), _Buffer()

    def __init__(self, pages, kv_heads, head_dim, page_size=16, fmt="int8", device="cuda"):
        if fmt not in FORMATS:
            raise ValueError("unknown cache format %r (int8 or fp8)" % (fmt,))
        self.pages, self.kv_heads, self.head_dim = int(pages), int(kv_heads), int(head_dim)
        self.page_size, self.fmt = int(page_size), fmt
        sizes = _lib.KvCacheDesc(self.pages, self.kv_heads, self.head_dim, self.page_size, FORMATS[fmt], None, None,
                                 None, None)
        n = ctypes.c_size_t()
        _raise(_lib.lib().convsel_kv_cache_bytes(ctypes.byref(sizes), ctypes.byref(n)), "KVCache")
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("KVCache lives on the GPU only")
        # Pages need no first value (their scale is set by the first write), but a read of one is then defined.
        self.k_codes = torch.zeros(n.value, dtype=torch.uint8, device=device)
        self.v_codes = torch.zeros(n.value, dtype=torch.uint8, device=device)
        # fp32 whatever torch's default type is: the library takes their addresses alone.
        self.k_scales = torch.zeros(self.pages, self.kv_heads, dtype=torch.float32, device=device)
        self.v_scales = torch.zeros(self.pages, self.kv_heads, dtype=torch.float32, device=device)
        self.device = self.k_codes.device
        # The cache as the library takes it; its buffers stay for the object's life.
        self._desc = ctypes.byref(_lib.KvCacheDesc(
            self.pages, self.kv_heads, self.head_dim, self.page_size, FORMATS[fmt], self.k_codes.data_ptr(),
            self.v_codes.data_ptr(), self.k_scales.data_ptr(), self.v_scales.data_ptr()))

    def _batch(self, what, table, lengths, offsets, tokens):
        """(descriptor, tensors it points into) of a call's sequences."""
        if table.dim() != 2:
            raise ValueError("%s: the block table must be [sequences][pages]" % what)
        n = table.shape[0]
        table = _ints(table, table.shape, what + ": the block table", self.device)
        lengths = _ints(lengths, (n,), what + ": lengths", self.device)
        offsets = _ints(offsets, (n + 1,), what + ": offsets", self.device)
        return ctypes.byref(_lib.KvBatchDesc(n, tokens, table.shape[1], table.data_ptr(), lengths.data_ptr(),
                                             offsets.data_ptr())), (table, lengths, offsets)

    def write(self, k, v, table, starts, offsets):
        """Quantises the packed tokens ``k`` and ``v`` ([tokens][kv_heads]
        [head_dim]) behind the ``starts[b]`` tokens that each sequence holds."""
        dt = _dtype_of("KVCache.write", k, v)
        k, v = _heads(k, "KVCache.write"), _heads(v, "KVCache.write")
        if k.shape != v.shape or k.shape[1:] != (self.kv_heads, self.head_dim) or k.device != self.device:
            raise ValueError("KVCache.write: k and v must be [tokens][%d][%d] on %s"
                             % (self.kv_heads, self.head_dim, self.device))
        b, keep = self._batch("KVCache.write", table, starts, offsets, k.shape[0])
        ks, vs = k.stride(), v.stride()
        _run("KVCache.write", _lib.lib().convsel_kv_write, self.device, self._desc, b, k.data_ptr(), v.data_ptr(), ks[0],
             ks[1], vs[0], vs[1], dt)

    def read(self, table, starts, offsets, tokens, dtype=torch.bfloat16):
        """(k, v) as values, [tokens][kv_heads][head_dim]: for each sequence the
        positions from ``starts[b]`` on, as many as ``offsets`` gives it;
        ``tokens`` is their total, offsets[-1]."""
        if dtype not in _DTYPES:
            raise ValueError("KVCache.read: unsupported dtype %s (float32 or bfloat16)" % dtype)
        b, keep = self._batch("KVCache.read", table, starts, offsets, int(tokens))
        k = torch.empty((tokens, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        _run("KVCache.read", _lib.lib().convsel_kv_read, self.device, self._desc, b, k.data_ptr(), v.data_ptr(),
             _DTYPES[dtype])
        return k, v


# ---- attention ------------------------------------------------------------------

def _window(window):
    """``window`` as the library takes it: one that no sequence can fill hides nothing, whatever its size."""
    return min(int(window), 2 ** 31 - 1)


@functools.lru_cache(maxsize=1024)
def _attention_plan(pages, kv_heads, head_dim, page_size, fmt, seqs, tokens, width, *sizes):
    """(descriptor by reference, workspace bytes) of a call of these sizes."""
    c = _lib.KvCacheDesc(pages, kv_heads, head_dim, page_size, fmt, None, None, None, None)
    b = _lib.KvBatchDesc(seqs, tokens, width, None, None, None)
    d, n = ctypes.byref(_lib.AttentionDesc(*sizes)), ctypes.c_size_t()
    _raise(_lib.lib().convsel_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), d, ctypes.byref(n)),
           "cached_attention")
    return d, n.value


def cached_attention(q, cache, table, lengths, offsets, causal=True, window=0, scale=None, out=None):
    """Attention of the packed queries ``q`` ([tokens][q_heads][head_dim]) over
    ``cache``: softmax(scale * q . K) V for each sequence, whose ``lengths[b]``
    cached tokens include the new ones (write them first).

    The queries of a sequence stand at its last positions; head h reads
    key/value head h // (q_heads // kv_heads).  ``causal`` hides later tokens,
    ``window`` > 0 all but the last ``window`` up to the query; a row with
    nothing left is zero.  ``scale`` is 1/sqrt(head_dim) by default.
    """
    dt = _dtype_of("cached_attention", q, out)
    q = _heads(q, "cached_attention")
    if q.shape[2] != cache.head_dim or q.shape[1] % cache.kv_heads or q.shape[1] == 0 or q.device != cache.device:
        raise ValueError("cached_attention: q must be [tokens][multiple of %d heads][%d] on %s"
                         % (cache.kv_heads, cache.head_dim, cache.device))
    if out is None:
        out = q.new_empty(q.shape)
    elif out.shape != q.shape or (out.stride(2) != 1 and q.shape[2] > 1):
        raise ValueError("cached_attention: out must have q's shape and a dense last dimension")
    b, keep = cache._batch("cached_attention", table, lengths, offsets, q.shape[0])
    qs, ys, c = q.stride(), out.stride(), cache._desc
    d, n = _attention_plan(cache.pages, cache.kv_heads, cache.head_dim, cache.page_size, FORMATS[cache.fmt],
                           table.shape[0], q.shape[0], table.shape[1], q.shape[1], dt, bool(causal), _window(window),
                           1.0 / math.sqrt(cache.head_dim) if scale is None else float(scale), qs[0], qs[1], ys[0],
                           ys[1])
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    _run("cached_attention", _lib.lib().convsel_attention, q.device, q.data_ptr(), c, b, out.data_ptr(), d,
         None if ws is None else ws.data_ptr(), n)
    return out


def describe_attention(cache, seqs, tokens, table_width, q_heads, dtype=torch.bfloat16, causal=True, window=0):
    """How the library runs cached_attention at these sizes, as one line."""
    b = _lib.KvBatchDesc(seqs, tokens, table_width, None, None, None)
    dim = cache.head_dim
    d = _lib.AttentionDesc(q_heads, _DTYPES[dtype], bool(causal), _window(window), 1.0, q_heads * dim, dim,
                           q_heads * dim, dim)
    buf = ctypes.create_string_buffer(512)
    _raise(_lib.lib().convsel_attention_describe(cache._desc, ctypes.byref(b), ctypes.byref(d), buf, len(buf)),
           "cached_attention")
    return buf.value.decode()


# ---- attention of prompts -------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _prompt_plan(q_at, k_at, v_at, *sizes):
    """(descriptor by reference, workspace bytes) of a call of these sizes, q, k and v at addresses of this alignment."""
    d, n = ctypes.byref(_lib.PromptDesc(*sizes)), ctypes.c_size_t()
    _raise(_lib.lib().convsel_prompt_attention_workspace_bytes(q_at, k_at, v_at, d, ctypes.byref(n)),
           "prompt_attention")
    return d, n.value


def prompt_attention(q, k, v, offsets, causal=True, window=0, scale=None, out=None):
    """Attention of whole prompts over their own keys and values, without a cache:
    softmax(scale * q . k) v for each of the packed sequences.

    ``q`` is [tokens][q_heads][head_dim] (up to 256), ``k`` and ``v`` are
    [tokens][kv_heads][head_dim], e.g. views of one fused projection;
    ``offsets`` (int32, [sequences + 1]) divides the tokens among the sequences.
    Head h reads key/value head h // (q_heads // kv_heads).  ``causal`` hides
    later tokens, ``window`` > 0 all but the last ``window`` up to the query;
    what they hide has no influence.  ``scale`` is 1/sqrt(head_dim) by default
    (2**127 at most in magnitude).
    Rows of ``out`` behind the last sequence are left as they were.
    """
    dt = _dtype_of("prompt_attention", q, k, v, out)
    q, k, v = (_heads(t, "prompt_attention") for t in (q, k, v))
    (t, hq, dim), hk = q.shape, k.shape[1]
    if k.shape != v.shape or k.shape[0] != t or k.shape[2] != dim or hk == 0 or hq == 0 or hq % hk:
        raise ValueError("prompt_attention: q %s, k %s and v %s do not belong together"
                         % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    if dim == 0:
        raise ValueError("prompt_attention: empty heads")
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("prompt_attention: offsets must be [sequences + 1]")
    offsets = _ints(offsets, offsets.shape, "prompt_attention: offsets", q.device)
    if out is None:
        out = q.new_empty(q.shape)
    elif out.shape != q.shape or (out.stride(2) != 1 and dim > 1):
        raise ValueError("prompt_attention: out must have q's shape and a dense last dimension")
    qs, ks, vs, ys = q.stride(), k.stride(), v.stride(), out.stride()
    qp, kp, vp = q.data_ptr(), k.data_ptr(), v.data_ptr()
    d, n = _prompt_plan(qp % 16, kp % 16, vp % 16, offsets.shape[0] - 1, t, hq, hk, dim, dt, bool(causal),
                        _window(window), 1.0 / math.sqrt(dim) if scale is None else float(scale), qs[0], qs[1], ks[0],
                        ks[1], vs[0], vs[1], ys[0], ys[1])
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    _run("prompt_attention", _lib.lib().convsel_prompt_attention, q.device, qp, kp, vp, offsets.data_ptr(),
         out.data_ptr(), d, None if ws is None else ws.data_ptr(), n)
    return out


def describe_prompt_attention(seqs, tokens, q_heads, kv_heads, head_dim, dtype=torch.bfloat16, causal=True, window=0):
    """How the library runs prompt_attention on dense tensors of these sizes, as one line."""
    q, k = (q_heads * head_dim, head_dim), (kv_heads * head_dim, head_dim)
    d = _lib.PromptDesc(seqs, tokens, q_heads, kv_heads, head_dim, _DTYPES[dtype], bool(causal), _window(window), 1.0,
                        *q, *k, *k, *q)
    buf = ctypes.create_string_buffer(512)
    _raise(_lib.lib().convsel_prompt_attention_describe(None, None, None, ctypes.byref(d), buf, len(buf)),
           "prompt_attention")
    return buf.value.decode()


# ---- linear on 8-bit codes --------------------------------------------------------

_CODES = -1


def _whole(n):
    """Bytes of a row of n codes in whole 16-byte units."""
    return (n + 15) // 16 * 16


@functools.lru_cache(maxsize=1024)
def _quantize_plan(*sizes):
    return ctypes.byref(_lib.QuantizeDesc(*sizes))


def quantize_rows(x):
    """``x`` coded by rows in 8 bits: (codes, scales), x = codes * scales[..., None]
    to within half a code.

    A row's scale (fp32) is its largest finite magnitude over 127, a code the
    quotient rounded to nearest even; infinities become the largest code of
    their sign and NaN 0.  Rows of codes lie in whole 16-byte units, zeros
    behind them, as ``linear_int8`` reads weights and rows best.
    """
    dt = _dtype_of("quantize_rows", x)
    if x.dim() < 1 or x.shape[-1] == 0:
        raise ValueError("quantize_rows: x must have rows, got shape %s" % (tuple(x.shape),))
    lead, i = x.shape[:-1], x.shape[-1]
    x2, ldx = _rows(x)
    m = x2.shape[0]
    codes = torch.empty((m, _whole(i)), dtype=torch.int8, device=x.device)
    scales = torch.empty(lead, dtype=torch.float32, device=x.device)
    if m:
        _run("quantize_rows", _lib.lib().convsel_quantize_rows, x.device, x2.data_ptr(), codes.data_ptr(),
             scales.data_ptr(), _quantize_plan(m, i, ldx, codes.shape[1], dt))
    codes = codes if codes.shape[1] == i else codes[:, :i]
    return (codes if x.dim() == 2 else codes.as_strided(x.shape, _row_strides(lead, codes.stride(0)))), scales


def _row_strides(lead, row):
    """Strides of rows ``row`` apart, in the order of the leading dimensions ``lead``."""
    strides = [1]
    for n in reversed(lead):
        strides.append(row)
        row *= n
    return strides[::-1]


@functools.lru_cache(maxsize=1024)
def _int8_plan(x_at, w_at, act, *sizes):
    """(descriptor by reference, workspace bytes) of a call of these sizes, x and w at addresses of this alignment."""
    if act not in ACTIVATIONS:
        raise ValueError("unknown activation %r (one of %s)" % (act, ", ".join(ACTIVATIONS)))
    *head, bias, residual = sizes
    d, n = ctypes.byref(_lib.LinearInt8Desc(*head, ACTIVATIONS[act], bias, residual)), ctypes.c_size_t()
    _raise(_lib.lib().convsel_linear_int8_workspace_bytes(x_at, w_at, d, ctypes.byref(n)), "linear_int8")
    return d, n.value


def _code_rows(w):
    """(w, ldw) with every row's last 16-byte unit in w's memory, as the kernels read it."""
    o, i = w.shape
    if i % 16 == 0 and w.is_contiguous():
        return w, i
    ldw = w.stride(0) if o > 1 else max(w.stride(0), i)
    if w.stride(1) == 1 or i == 1:
        end = (o - 1) * ldw + (_whole(i) if ldw % 16 == 0 and w.data_ptr() % 16 == 0 else i)
        if ldw >= i and w.untyped_storage().nbytes() - w.storage_offset() >= end:
            return w, ldw
    rows = torch.empty((o, _whole(i)), dtype=torch.int8, device=w.device)
    rows[:, :i] = w
    return rows, rows.shape[1]


def _scales(t, shape, what, device):
    if t.dtype is not torch.float32 or t.shape != shape or t.device != device:
        raise ValueError("%s must be a float32 tensor of shape %s on %s" % (what, tuple(shape), device))
    return t if t.is_contiguous() else t.contiguous()


def linear_int8(x, w, w_scale, b=None, act="none", residual=None, x_scale=None, dtype=None, out=None):
    """``act((x @ w.T) * scales + b) + residual`` over the last dimension of
    ``x``, with the products and their sum in whole numbers.

    ``w`` ([out_features][in_features]) and ``w_scale`` are the codes and scales of the
    weights (``quantize_rows(weight)``).  ``x`` is float32 or bfloat16, coded
    by rows within the call, or codes with their ``x_scale``
    (``quantize_rows(x)``, once for several layers).  The result, ``b``,
    ``residual`` and ``out`` are of ``dtype``: x's, or bfloat16 for codes, by
    default.  ``act`` is as in ``linear``; ``out`` may be ``residual`` itself.
    """
    codes = x.dtype is torch.int8
    if not x.is_cuda:
        raise ValueError("linear_int8 runs on the GPU only: move its tensors to a HIP device")
    dev = x.device
    x_dt = _CODES if codes else _dtype_of("linear_int8", x)
    if dtype is None:
        dtype = out.dtype if out is not None else torch.bfloat16 if codes else x.dtype
    dt = _DTYPES.get(dtype)
    if dt is None:
        raise ValueError("linear_int8: unsupported dtype %s (float32 or bfloat16)" % dtype)
    for t in (b, residual, out):
        if t is not None and (t.dtype is not dtype or t.device != dev):
            raise ValueError("linear_int8: b, residual and out must be %s on %s" % (dtype, dev))
    if w.dtype is not torch.int8 or w.device != dev:
        raise ValueError("linear_int8: w must hold int8 codes on %s" % dev)
    if x.dim() < 1 or w.dim() != 2 or x.shape[-1] != w.shape[1]:
        raise ValueError("linear_int8: input features of x %s and weight %s differ" % (tuple(x.shape), tuple(w.shape)))
    if codes != (x_scale is not None):
        raise ValueError("linear_int8: x_scale comes with an x of codes, and only then")
    o, i = w.shape
    if i == 0 or o == 0:
        raise ValueError("linear_int8: empty weight")
    w_scale = _scales(w_scale, (o,), "linear_int8: w_scale", dev)
    if b is not None and tuple(b.shape) != (o,):
        raise ValueError("linear_int8: bias must hold %d values" % o)
    shape = x.shape[:-1] + (o,)
    if codes:
        x_scale = _scales(x_scale, x.shape[:-1], "linear_int8: x_scale", dev)
    if residual is not None and residual.shape != shape:
        raise ValueError("linear_int8: residual must have shape %s" % (tuple(shape),))
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
    elif out.shape != shape:
        raise ValueError("linear_int8: out must have shape %s" % (tuple(shape),))
    if out.numel() == 0:
        return out
    x2, ldx = _rows(x)
    y2, ldy = _rows(out)
    if y2.data_ptr() != out.data_ptr():
        raise ValueError("linear_int8: out must be a view of rows with a dense last dimension")
    r2, ldr = (None, 0) if residual is None else _rows(residual)
    w, ldw = _code_rows(w)
    b = None if b is None else b.contiguous()
    xp, wp = x2.data_ptr(), w.data_ptr()
    d, n = _int8_plan(xp % 16, wp % 16, act, x2.shape[0], i, o, ldx, ldw, ldr, ldy, x_dt, dt, b is not None,
                      r2 is not None)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _run("linear_int8", _lib.lib().convsel_linear_int8, dev, xp, None if x_scale is None else x_scale.data_ptr(), wp,
         w_scale.data_ptr(), None if b is None else b.data_ptr(), None if r2 is None else r2.data_ptr(), y2.data_ptr(),
         d, None if ws is None else ws.data_ptr(), n)
    return out


def describe_linear_int8(m, in_features, out_features, dtype=torch.bfloat16, codes=False, act="none", bias=False,
                         residual=False):
    """How the library runs this layer on rows as ``quantize_rows`` lays them out, as one line."""
    wide = _whole(in_features)
    d = _lib.LinearInt8Desc(m, in_features, out_features, wide if codes else in_features, wide, out_features,
                            out_features, _CODES if codes else _DTYPES[dtype], _DTYPES[dtype], ACTIVATIONS[act], bias,
                            residual)
    buf = ctypes.create_string_buffer(512)
    _raise(_lib.lib().convsel_linear_int8_describe(None, None, ctypes.byref(d), buf, len(buf)), "linear_int8")
    return buf.value.decode()


# ---- logits -----------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _logits_plan(*sizes):
    return ctypes.byref(_lib.LogitsDesc(*sizes))


def adjust_logits(logits, history=None, offsets=None, prompt_lengths=None, repetition=None, presence=None,
                  frequency=None, bias=None, mask=None, out=None):
    """``logits`` ([rows][vocabulary]) as a token is chosen from: with the
    penalties of the tokens that each row has seen, biases and a mask.

    ``history`` (int32) holds the rows' tokens, packed by ``offsets`` (int32,
    [rows + 1]); the first ``prompt_lengths[b]`` (int32; none by default) of a row
    are its prompt, the others were generated.  In this order, for a token t:

    * in the history: z / repetition[b] where z > 0, else z * repetition[b];
    * generated c > 0 times: z - (frequency[b] * c + presence[b]);
    * z + bias[t], or bias[b][t];
    * -inf where bit t % 32 of word t // 32 of ``mask`` (int32, [rows][words] or
      [words]) is clear.

    Penalties and biases are float32.  ``out`` may be ``logits`` itself.
    """
    dt = _dtype_of("adjust_logits", logits, out)
    if logits.dim() != 2 or logits.shape[1] == 0:
        raise ValueError("adjust_logits: logits must be [rows][vocabulary], got shape %s" % (tuple(logits.shape),))
    (n, vocab), dev = logits.shape, logits.device
    if (history is None) != (offsets is None):
        raise ValueError("adjust_logits: history and offsets come together")
    penalties = (repetition, presence, frequency)
    if history is None and (prompt_lengths is not None or any(p is not None for p in penalties)):
        raise ValueError("adjust_logits: penalties need a history")
    tokens = 0
    if history is not None:
        if history.dim() != 1:
            raise ValueError("adjust_logits: the history must be packed in one dimension")
        history = _ints(history, history.shape, "adjust_logits: history", dev)
        offsets = _ints(offsets, (n + 1,), "adjust_logits: offsets", dev)
        tokens = history.shape[0]
        if prompt_lengths is not None:
            prompt_lengths = _ints(prompt_lengths, (n,), "adjust_logits: prompt_lengths", dev)
        repetition, presence, frequency = (
            None if p is None else _scales(p, (n,), "adjust_logits: a penalty", dev) for p in penalties)
        if tokens == 0:  # an empty tensor has no address
            history = offsets
    ldbias = ldmask = 0
    if bias is not None:
        if bias.dim() not in (1, 2):
            raise ValueError("adjust_logits: bias must be [vocabulary] or [rows][vocabulary]")
        bias = _scales(bias, (vocab,) if bias.dim() == 1 else (n, vocab), "adjust_logits: bias", dev)
        ldbias = 0 if bias.dim() == 1 else vocab
    if mask is not None:
        words = (vocab + 31) // 32
        if mask.dim() not in (1, 2):
            raise ValueError("adjust_logits: mask must be [words] or [rows][words]")
        mask = _ints(mask, (words,) if mask.dim() == 1 else (n, words), "adjust_logits: mask", dev)
        ldmask = 0 if mask.dim() == 1 else words
    if logits.stride(1) != 1 and vocab > 1 or logits.stride(0) < vocab and n > 1:
        logits = logits.contiguous()
    if out is None:
        out = logits.new_empty((n, vocab))
    elif out.shape != logits.shape or (out.stride(1) != 1 and vocab > 1):
        raise ValueError("adjust_logits: out must have the logits' shape and a dense last dimension")
    if n == 0:
        return out
    d = _logits_plan(n, vocab, tokens, logits.stride(0) if n > 1 else vocab, out.stride(0) if n > 1 else vocab, ldbias,
                     ldmask, dt)
    _run("adjust_logits", _lib.lib().convsel_adjust_logits, dev, logits.data_ptr(),
         *(None if t is None else t.data_ptr() for t in (history, offsets, prompt_lengths, repetition, presence,
                                                         frequency, bias, mask)), out.data_ptr(), d)
    return out
