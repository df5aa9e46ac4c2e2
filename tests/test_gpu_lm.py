"""GPU checks of the decoder operators against their 64-bit forms: each at the
sizes, strides, masks and device-side numbers where it can go wrong.  Bounds
come from the roundings that the operators state (ref_lm.py)."""
import math

import numpy as np
import pytest
import torch

import ref_lm as ref
from gpu_util import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2410_08300_amd as cs  # noqa: E402

DEV = torch.device("cuda:0")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def within(got, want, bound, what):
    got, want, bound = (np.asarray(a.double().cpu() if torch.is_tensor(a) else a, dtype=np.float64)
                        for a in (got, want, bound))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = np.abs(got - want)
    over = ~(err <= bound)
    assert not over.any(), "%s: %d of %d beyond the bound, worst %.3g of %.3g" % (
        what, over.sum(), over.size, err[over].max() if np.isfinite(err[over]).any() else float("nan"),
        bound[over].flat[0])


# ---- linear -----------------------------------------------------------------

# m, in, out: single rows, few rows, one more or less than tiles, odd widths, long sums, many rows.
LINEAR_SIZES = [(1, 64, 48), (1, 4096, 512), (1, 8200, 129), (2, 1, 1), (3, 7, 5), (4, 1000, 333), (7, 72, 1001),
                (15, 136, 64), (16, 512, 96), (17, 520, 130), (33, 256, 255), (63, 65, 64), (64, 64, 64),
                (65, 1032, 257), (100, 129, 128), (128, 2048, 256), (129, 320, 384), (200, 4104, 120), (255, 96, 513),
                (256, 256, 256), (257, 264, 264), (513, 512, 520), (1000, 200, 72), (2050, 128, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", LINEAR_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_sizes(size, dtype):
    m, i, o = size
    say("case linear", size, dtype)
    g, dt = gen(m * 7 + i * 3 + o), DT[dtype]
    x = torch.randn(m, i, generator=g, device=DEV).to(dt)
    w = (torch.randn(o, i, generator=g, device=DEV) / i ** 0.5).to(dt)
    b = torch.randn(o, generator=g, device=DEV).to(dt)
    r = torch.randn(m, o, generator=g, device=DEV).to(dt)
    for activation, bias, res in (("none", None, None), ("gelu_tanh", b, r), ("relu", b, None)):
        y = cs.linear(x, w, bias, act=activation, residual=res)
        want, bound = ref.linear(x, w, bias, activation, res)
        within(y, want, bound + ref.half_ulp(dt) * want.abs() * 1.01, "linear %s %s" % (size, activation))


# One case for each tile and way of cutting it, with the kernels that it must reach.
TILE_SIZES = [(4000, 72, 4001, "tile=128x128 split=1"), (3999, 200, 4000, "tile=128x128 split=1"),
              (2000, 136, 2100, "tile=128x128 split=1"), (2050, 1030, 2048, "linear_pack_kernel;linear_tiles_kernel tile=128x128 split=1"),
              (1030, 8200, 2052, "tile=128x128 split="), (100, 2056, 130, "tile=64x64 split="),
              (500, 260, 1000, "linear_pack_kernel;linear_tiles_kernel tile=64x64 split=1"), (1111, 100, 999, "tile=64x64 split=1")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", TILE_SIZES, ids=lambda s: "x".join(map(str, s[:3])))
def test_linear_in_every_tile(size, dtype):
    m, i, o, runs = size
    dt = DT[dtype]
    say("case linear tile", size, dtype, cs.describe_linear(m, i, o, dt))
    if dtype == "bf16":
        assert runs in cs.describe_linear(m, i, o, dt)
    g = gen(m + i)
    x = torch.randn(m, i, generator=g, device=DEV).to(dt)
    w = (torch.randn(o, i, generator=g, device=DEV) / i ** 0.5).to(dt)
    b = torch.randn(o, generator=g, device=DEV).to(dt)
    r = torch.randn(m, o, generator=g, device=DEV).to(dt)
    whole = torch.full((m + 2, o + 6), 7.0, device=DEV, dtype=dt)
    y = whole[1:-1, 2:o + 2]
    cs.linear(x, w, b, act="silu", residual=r, out=y)
    # The reference on the GPU in 64 bits: its own roundings are nothing here.
    xd, wd = x.double(), w.double()
    z = xd @ wd.T.contiguous() + b.double()
    mag = xd.abs() @ wd.abs().T.contiguous() + b.double().abs()
    want = z / (1 + torch.exp(-z))
    bound = (i + 8) * 2.0 ** -24 * 1.13 * mag + 16 * 2.0 ** -24 * want.abs()
    want = want + r.double()
    bound = bound + (2.0 ** -24 + ref.half_ulp(dt) * 1.01) * want.abs()
    assert bool(((y.double() - want).abs() <= bound).all())
    inside = torch.zeros_like(whole, dtype=torch.bool)
    inside[1:-1, 2:o + 2] = True
    assert bool((whole[~inside] == 7.0).all())
    assert torch.equal(cs.linear(x, w, b, act="silu", residual=r), y)


# Few rows: by rows, read on 16 bytes and on none, and in tiles where outputs are few; rows that would be copied first.
FEW_ROWS = [("f32", 15, 2041, 300, "linear_rows_kernel"), ("bf16", 5, 1363, 1867, "linear_rows_kernel"),
            ("bf16", 3, 67, 33, "linear_rows_kernel"), ("f32", 7, 14088, 41, "linear_tiles_kernel;linear_join_kernel"),
            ("bf16", 5, 11648, 68, "linear_tiles_kernel;linear_join_kernel"),
            ("f32", 29, 2282, 1496, "linear_rows_kernel"), ("bf16", 28, 717, 119, "linear_rows_kernel")]


@pytest.mark.parametrize("size", FEW_ROWS, ids=lambda s: "%s-%dx%dx%d" % s[:4])
def test_linear_of_few_rows(size):
    dtype, m, i, o, runs = size
    dt = DT[dtype]
    say("case linear few", size, cs.describe_linear(m, i, o, dt))
    assert runs in cs.describe_linear(m, i, o, dt)
    g = gen(m * o)
    # Behind the operands lies NaN: nothing past a row's end may count.
    x = torch.full((m * i + 64,), float("nan"), device=DEV, dtype=dt)[:m * i].view(m, i)
    w = torch.full((o * i + 64,), float("nan"), device=DEV, dtype=dt)[:o * i].view(o, i)
    x.copy_(torch.randn(m, i, generator=g, device=DEV))
    w.copy_(torch.randn(o, i, generator=g, device=DEV))
    b, r = torch.randn(o, generator=g, device=DEV).to(dt), torch.randn(m, o, generator=g, device=DEV).to(dt)
    want, bound = ref.linear(x, w, b, "gelu_tanh", r)
    within(cs.linear(x, w, b, act="gelu_tanh", residual=r), want, bound + ref.half_ulp(dt) * want.abs() * 1.01,
           "few %s" % (size,))


# The kernel for tiles of 256: a cut last k-tile and none, rows and outputs that end inside a tile, copied operands, parts.
BIG_TILES = [("bf16", 3999, 720, 4000, "linear_tiles256_kernel tile=256x256 split=1"),
             ("f32", 3999, 720, 4000, "linear_tiles_kernel tile=256x256 split=1"),
             ("bf16", 3850, 1030, 4001, "linear_pack_kernel;linear_tiles256_kernel tile=256x256 split=1"),
             ("f32", 3850, 1023, 4001, "linear_pack_kernel;linear_tiles_kernel tile=256x256 split=1"),
             ("bf16", 700, 4096, 4096, "tile=256x256 split=5"), ("bf16", 1500, 4104, 4096, "tile=256x256 split=2")]


@pytest.mark.parametrize("size", BIG_TILES, ids=lambda s: "%s-%dx%dx%d" % s[:4])
def test_linear_in_tiles_of_256(size):
    dtype, m, i, o, runs = size
    dt = DT[dtype]
    say("case linear tile 256", size, cs.describe_linear(m, i, o, dt))
    assert runs in cs.describe_linear(m, i, o, dt)
    g = gen(m + i)
    x, w = torch.randn(m, i, generator=g, device=DEV).to(dt), torch.randn(o, i, generator=g, device=DEV).to(dt)
    b, r = torch.randn(o, generator=g, device=DEV).to(dt), torch.randn(m, o, generator=g, device=DEV).to(dt)
    y = cs.linear(x, w, b, act="silu", residual=r)
    # Rows from the first, middle and last tiles, and the outputs of all.
    rows = torch.tensor(sorted({0, 1, 31, 127, 128, 255, 256, 300, 511, m // 2, m - 2, m - 1}), device=DEV)
    want, bound = ref.linear(x[rows], w, b, "silu", r[rows])
    within(y[rows], want, bound + ref.half_ulp(dt) * want.abs() * 1.01, "linear 256 %s" % (size,))
    # Every other row against the same sums in fp32 by torch's own order: no row may be another's.
    near = torch.nn.functional.silu(x.float() @ w.float().T + b.float()) + r.float()
    assert float((y.float() - near).abs().max()) <= 2.0 ** -6 * float(near.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("activation", list(cs.ACTIVATIONS))
def test_linear_activations_over_their_range(activation, dtype):
    say("case linear activation", activation, dtype)
    dt = DT[dtype]
    z = torch.cat([torch.linspace(-40, 40, 4001, device=DEV), torch.tensor([0., -0., 1e-20, -1e-20, 300., -300.],
                                                                           device=DEV)]).to(dt)[:, None]
    y = cs.linear(z, torch.ones(1, 1, device=DEV, dtype=dt), act=activation)
    want, bound = ref.linear(z, torch.ones(1, 1), None, activation)
    # gelu's 1 + erf cancels on the left: 2^-24 of 1, times z/2; the tanh and silu forms lose the exponential's
    # argument error, 2^-24 of the argument (a cube), relative.
    u = z.double().cpu().abs()
    slack = 4 * 2.0 ** -24 * u + 8 * 2.0 ** -24 * (1 + u ** 3 * 0.08) * want.abs().clamp(max=64) + 1e-37
    within(y, want, bound + slack + ref.half_ulp(dt) * want.abs() * 1.01, activation)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_linear_strided_rows_leading_dims_and_guards(m, dtype):
    say("case linear strided", m, dtype)
    g, dt = gen(m), DT[dtype]
    i, o = 72, 104
    wide = torch.randn(m, 3, i + 5, generator=g, device=DEV).to(dt)
    w = torch.randn(o, i, generator=g, device=DEV).to(dt)
    x = wide[:, 1, 3:3 + i]  # rows of stride 3 (i + 5) from an address of no 16 bytes
    res = torch.randn(m, o + 9, generator=g, device=DEV).to(dt)[:, 4:4 + o]
    whole = torch.full((m + 2, o + 11), 7.0, device=DEV, dtype=dt)
    out = whole[1:m + 1, 6:6 + o]
    want, bound = ref.linear(x, w, None, "silu", res)
    y = cs.linear(x, w, act="silu", residual=res, out=out)
    assert y.data_ptr() == out.data_ptr()
    within(out, want, bound + ref.half_ulp(dt) * want.abs() * 1.01, "strided")
    inside = torch.zeros_like(whole, dtype=torch.bool)
    inside[1:m + 1, 6:6 + o] = True
    assert bool((whole[~inside] == 7.0).all()), "wrote outside its rows"
    # three leading dimensions, and an empty batch
    x3 = x.reshape(1, m, 1, i)
    assert torch.equal(cs.linear(x3, w, act="silu", residual=res.reshape(1, m, 1, o)).view(m, o), out)
    assert cs.linear(x[:0], w).shape == (0, o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_many_rows_that_tiles_cannot_address(dtype):
    """Rows further apart than a tile's offsets reach, and operands that start on no 16 bytes, through the C entry."""
    dt, m, i, o = DT[dtype], 37, 96, 50
    say("case linear rows", dtype)
    far = (1 << 31) // 256 // dt.itemsize + 8
    g = gen(9)
    base = torch.empty(m * far + 64, device=DEV, dtype=dt)
    x = base.as_strided((m, i), (far, 1), 16)
    x.copy_(torch.randn(m, i, generator=g, device=DEV))
    w = torch.randn(o, i, generator=g, device=DEV).to(dt)
    r = torch.randn(m, o, generator=g, device=DEV).to(dt)
    want, bound = ref.linear(x, w, None, "relu", r)
    bound = bound + ref.half_ulp(dt) * want.abs() * 1.01
    within(cs.linear(x, w, act="relu", residual=r), want, bound, "far rows")
    lib = cs._lib.lib()
    for shift in (1, 3):
        xs = torch.empty(m * i + shift, device=DEV, dtype=dt)[shift:].view(m, i).copy_(x)
        ws = torch.empty(o * i + shift, device=DEV, dtype=dt)[shift:].view(o, i).copy_(w)
        y = torch.empty(m, o, device=DEV, dtype=dt)
        d, n = cs.lm._linear_plan(m, i, o, i, o, o, cs.lm._DTYPES[dt], "relu", False, True)
        space = torch.empty(max(n, 1), device=DEV, dtype=torch.uint8)
        st = lib.convsel_linear(xs.data_ptr(), ws.data_ptr(), None, r.data_ptr(), y.data_ptr(), d, space.data_ptr(), n,
                                torch.cuda.current_stream().cuda_stream)
        assert st == 0
        within(y, want, bound, "shifted by %d" % shift)


def test_linear_updates_its_residual_in_place():
    for m in (1, 9, 70, 300):
        x, w = torch.randn(m, 256, device=DEV).bfloat16(), torch.randn(192, 256, device=DEV).bfloat16()
        r = torch.randn(m, 192, device=DEV).bfloat16()
        want = cs.linear(x, w, residual=r)
        got = r.clone()
        cs.linear(x, w, residual=got, out=got)
        assert torch.equal(got, want), m


@pytest.mark.parametrize("m", [1, 12, 100, 400])
def test_linear_carries_infinities_and_nan_in_their_own_rows(m):
    x = torch.randn(m, 320, device=DEV)
    w = torch.randn(200, 320, device=DEV)
    for dt in (torch.float32, torch.bfloat16):
        a, c = x.to(dt), w.to(dt)
        clean = cs.linear(a, c, act="relu")
        bad = a.clone()
        bad[m // 2, 5] = float("nan")
        y = cs.linear(bad, c, act="relu")
        assert bool(y[m // 2].isnan().all())
        keep = torch.arange(m, device=DEV) != m // 2
        assert torch.equal(y[keep], clean[keep])


def test_linear_is_the_same_every_time():
    for m, i, o in ((1, 4096, 4096), (8, 8192, 512), (48, 4096, 256), (300, 1000, 520)):
        x, w = torch.randn(m, i, device=DEV).bfloat16(), torch.randn(o, i, device=DEV).bfloat16()
        first = cs.linear(x, w)
        for _ in range(5):
            assert torch.equal(cs.linear(x, w), first), (m, i, o)


# ---- norm and rotation ---------------------------------------------------------

def rope_tables(rows, rotary):
    freq = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().to(DEV), angle.sin().float().to(DEV)


ROPE_CASES = [  # tokens, q heads, k heads, dim, rotary, interleaved, norm, weights
    (1, 8, 2, 128, 128, False, "rms", True), (5, 3, 1, 64, 64, True, "rms", True), (7, 4, 4, 80, 32, False, "rms", False),
    (33, 2, 2, 96, 96, True, "none", True), (3, 1, 1, 2, 2, False, "rms", True), (9, 5, 0, 256, 64, False, "rms", True),
    (4, 0, 3, 192, 96, True, "none", False), (6, 2, 1, 7, 4, False, "rms", True), (2, 2, 2, 1024, 1024, False, "rms", True),
    (65, 6, 3, 32, 0, False, "rms", True), (3, 2, 2, 100, 50, False, "rms", True), (257, 2, 1, 128, 64, True, "rms", True),
    (4, 3, 2, 512, 512, True, "rms", True), (2, 1, 1, 1, 0, False, "rms", True), (6, 33, 5, 128, 128, False, "rms", True),
    (4, 40, 1, 64, 32, False, "rms", True), (2, 9, 9, 72, 16, False, "none", True), (8, 2, 17, 256, 256, True, "rms", False),
    (4, 7, 3, 1024, 512, False, "rms", True), (2, 3, 3, 8, 8, True, "rms", True), (130, 5, 2, 96, 0, False, "none", False),
    (2050, 3, 1, 64, 64, True, "rms", True), (2051, 9, 2, 128, 64, False, "rms", True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROPE_CASES, ids=lambda c: "-".join(map(str, c)))
def test_qk_norm_rope(case, dtype):
    say("case rope", case, dtype)
    t, hq, hk, d, rot, inter, norm, weights = case
    g, dt = gen(t + d), DT[dtype]
    # A fused projection with a few columns more than it needs, from an odd column on in one case of two.
    lead = 3 if t % 2 else 0
    fused = torch.randn(t, (hq + 2 * hk) * d + 8, generator=g, device=DEV).to(dt) * 2
    q = fused[:, lead:lead + hq * d].view(t, hq, d)
    k = fused[:, lead + hq * d:lead + (hq + hk) * d].view(t, hk, d)
    qw = torch.randn(d, generator=g, device=DEV).to(dt) if weights else None
    kw = torch.randn(d, generator=g, device=DEV).to(dt) if weights else None
    cos, sin = rope_tables(500, rot) if rot else (None, None)
    pos = torch.randint(0, 500, (t,), generator=g, device=DEV, dtype=torch.int32)
    qo, ko = cs.qk_norm_rope(q, k, pos, cos, sin, qw, kw, eps=1e-5, norm=norm, interleaved=inter)
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        want, mag = ref.norm_rope(x, w, pos.tolist(), None if cos is None else cos.cpu(),
                                  None if sin is None else sin.cpu(), 1e-5, norm == "rms", inter)
        # The norm: a sum of d squares, a root, a quotient and two products; the rotation: three roundings.
        bound = ((d / 2 + 16) * 2.0 ** -24) * mag + ref.half_ulp(dt) * want.abs() * 1.01
        within(got, want, bound, "rope %s" % (case,))
    # The same in place, in the fused projection itself: nothing else of it changes.
    before = fused.clone()
    cs.qk_norm_rope(q, k, pos, cos, sin, qw, kw, eps=1e-5, norm=norm, interleaved=inter, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    mask = torch.ones(fused.shape[1], dtype=torch.bool, device=DEV)
    mask[lead:lead + (hq + hk) * d] = False
    assert torch.equal(fused[:, mask], before[:, mask])


@pytest.mark.parametrize("dim,rot", [(128, 128), (80, 32), (7, 4)])
def test_positions_outside_the_tables_are_nan_and_read_nothing(dim, rot):
    cos, sin = rope_tables(10, rot)
    q = torch.randn(6, 2, dim, device=DEV)
    pos = ints([0, 9, 10, -1, 2 ** 31 - 1, -2 ** 31])
    qo, ko = cs.qk_norm_rope(q, q[:, :1], pos, cos, sin)
    for o in (qo, ko):
        assert bool(o[:2].isfinite().all()) and bool(o[2:].isnan().all())


@pytest.mark.parametrize("dim,rot,inter", [(128, 64, False), (128, 32, True), (80, 16, False), (7, 4, False)])
def test_infinities_stay_where_nothing_turns_and_with_their_partners(dim, rot, inter):
    cos, sin = rope_tables(64, rot)
    pos = ints([3, 5])
    for dt in (torch.float32, torch.bfloat16):
        x = torch.randn(2, 3, dim, device=DEV).to(dt)
        bad = x.clone()
        bad[0, 1, dim - 1] = float("inf")
        bad[1, 2, 0] = float("inf")
        want, _ = cs.qk_norm_rope(x, x[:, :1], pos, cos, sin, norm="none", interleaved=inter)
        got, _ = cs.qk_norm_rope(bad, x[:, :1], pos, cos, sin, norm="none", interleaved=inter)
        assert float(got[0, 1, dim - 1]) == float("inf")
        other = 1 if inter else rot // 2
        assert not bool(got[1, 2, [0, other]].isfinite().any())
        same = torch.ones_like(x, dtype=torch.bool)
        same[0, 1, dim - 1] = same[1, 2, 0] = same[1, 2, other] = False
        assert torch.equal(got[same], want[same])


def test_heads_of_zeros_and_head_major_strides():
    cos, sin = rope_tables(64, 64)
    pos = ints(list(range(5)))
    z = torch.zeros(5, 2, 64, device=DEV, dtype=torch.bfloat16)
    qo, ko = cs.qk_norm_rope(z, z, pos, cos, sin)
    assert bool((qo == 0).all()) and bool((ko == 0).all())
    x = torch.randn(3, 5, 64, device=DEV).bfloat16()  # head-major
    y = torch.empty_like(x)
    cs.qk_norm_rope(x.transpose(0, 1), x.transpose(0, 1)[:, :2], pos, cos, sin, q_out=y.transpose(0, 1))
    want, _ = cs.qk_norm_rope(x.transpose(0, 1).contiguous(), x.transpose(0, 1)[:, :2].contiguous(), pos, cos, sin)
    assert torch.equal(y.transpose(0, 1), want)


# ---- cache --------------------------------------------------------------------

def fresh(pages, heads, dim, page, fmt):
    """A cache whose memory held other things before, and its definition."""
    c = cs.KVCache(pages, heads, dim, page_size=page, fmt=fmt)
    for t in (c.k_codes, c.v_codes):
        t.fill_(0xFF)  # NaN in e4m3
    for t in (c.k_scales, c.v_scales):
        t.fill_(float("nan"))
    return c, ref.Cache(pages, heads, dim, page, fmt)


def values(cache, table, starts, counts, name):
    out = []
    for b in range(len(starts)):
        for p in range(starts[b], starts[b] + counts[b]):
            v = cache.value(name, table, b, p)
            out.append(np.zeros(cache.codes[name].shape[1::2]) if v is None else v)
    return np.stack(out) if out else np.zeros((0,) + cache.codes[name].shape[1::2])


def offsets_of(counts):
    return [0] + list(np.cumsum(counts).tolist())


# heads, dim, page, then writes: for each, how many tokens every sequence gets.
CACHE_CASES = [
    (2, 128, 16, [[1, 1, 1]] * 5),                        # generation from empty pages
    (3, 64, 32, [[37, 0, 16], [1, 5, 1], [0, 30, 200]]),  # prompts of unlike lengths, an idle sequence, page ends
    (1, 80, 64, [[63], [1], [1], [129]]),                 # a padded row, the last row of a page, the first of the next
    (2, 7, 16, [[15, 17], [2, 2]]),
    (1, 1, 128, [[130], [3]]),
    (2, 256, 16, [[33, 1], [15, 16]]),
    (1, 96, 128, [[1, 127, 128, 129], [3, 1, 1, 1], [200, 0, 0, 1]]),
    (4, 32, 64, [[0, 0], [64, 65], [0, 1]]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("case", CACHE_CASES, ids=lambda c: "h%d-d%d-p%d" % c[:3])
def test_cache_write_and_read(case, fmt, dtype):
    heads, dim, page, writes = case
    say("case cache", case, fmt, dtype)
    g, dt = gen(dim + page), DT[dtype]
    seqs = len(writes[0])
    total = np.sum(writes, axis=0)
    width = int(max(total) + page - 1) // page + 1
    pages = seqs * width + 2
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    table = [order[b * width:(b + 1) * width] for b in range(seqs)]
    cache, want = fresh(pages, heads, dim, page, fmt)
    held = [0] * seqs
    for step, counts in enumerate(writes):
        off = offsets_of(counts)
        # Magnitudes that grow and shrink from call to call, so that scales grow in some pages and not in others.
        gain = (0.1, 3.0, 1.0, 20.0, 0.5)[step % 5]
        kv = torch.randn(off[-1], 2, heads, dim + 3, generator=g, device=DEV).to(dt) * gain
        k, v = kv[:, 0, :, 1:dim + 1], kv[:, 1, :, :dim]  # strided, from odd addresses
        cache.write(k, v, ints(table), ints(held), ints(off))
        want.write(k, v, table, held, off)
        held = [h + n for h, n in zip(held, counts)]
        k2, v2 = cache.read(ints(table), ints([0] * seqs), ints(offsets_of(held)), sum(held), dtype=torch.float32)
        for got, name in ((k2, "k"), (v2, "v")):
            exact = values(want, table, [0] * seqs, held, name).astype(np.float32)  # one rounded product
            assert np.array_equal(got.cpu().numpy(), exact), "%s after write %d" % (name, step)
    # A read from the middle, rounded to bf16.
    mid = [h // 3 for h in held]
    counts = [h - s for h, s in zip(held, mid)]
    k2, _ = cache.read(ints(table), ints(mid), ints(offsets_of(counts)), sum(counts))
    exact = values(want, table, mid, counts, "k").astype(np.float32)
    assert torch.equal(k2.cpu(), torch.from_numpy(exact).bfloat16())


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_cache_takes_infinities_nan_zeros_and_tiny_numbers(fmt):
    cache, want = fresh(4, 1, 32, 16, fmt)
    x = torch.randn(48, 1, 32, device=DEV)
    x[3, 0, 4], x[5, 0, 6], x[7, 0, 8] = float("inf"), float("-inf"), float("nan")
    x[16:32] = 0
    x[32:48] *= 1e-36
    table, off = [[2, 0, 3]], [0, 48]
    cache.write(x, x * 2, ints(table), ints([0]), ints(off))
    want.write(x, x * 2, table, [0], off)
    k, v = cache.read(ints(table), ints([0]), ints(off), 48, dtype=torch.float32)
    assert np.array_equal(k.cpu().numpy(), values(want, table, [0], [48], "k").astype(np.float32))
    assert np.array_equal(v.cpu().numpy(), values(want, table, [0], [48], "v").astype(np.float32))
    top = float(x[:16][x[:16].isfinite()].abs().max())
    assert float(k[3, 0, 4]) == pytest.approx(top, rel=1e-6) and float(k[5, 0, 6]) == pytest.approx(-top, rel=1e-6)
    assert float(k[7, 0, 8]) == 0 and bool((k[16:32] == 0).all())


def test_cache_skips_pages_it_does_not_have_and_rows_past_the_table():
    cache, want = fresh(3, 2, 64, 16, "int8")
    table = [[-1, 1, 3], [2, 2 ** 31 - 1, 0]]
    off = [0, 60, 100]  # the first sequence runs past its table, the second names no page in between
    x = torch.randn(100, 2, 64, device=DEV).bfloat16()
    codes = [cache.k_codes.clone(), cache.v_codes.clone()]
    cache.write(x, x, ints(table), ints([0, 0]), ints(off))
    want.write(x, x, table, [0, 0], off)
    k, v = cache.read(ints(table), ints([0, 0]), ints(off), 100, dtype=torch.float32)
    exact = values(want, table, [0, 0], [60, 40], "k").astype(np.float32)
    assert np.array_equal(k.cpu().numpy(), exact) and np.array_equal(v.cpu().numpy(), exact)
    # Page 0 got rows 0..7 of the second sequence's third page: the other rows keep what they held.
    rows = cache.k_codes.view(3, 2, 16, 64)
    assert torch.equal(rows[0, :, 8:], codes[0].view(3, 2, 16, 64)[0, :, 8:])
    # Reads before a sequence and far behind its table are zeros.
    k, v = cache.read(ints(table), ints([-5, 2 ** 31 - 30]), ints([0, 5, 25]), 25, dtype=torch.float32)
    assert bool((k == 0).all()) and bool((v == 0).all())


def test_cache_offsets_out_of_range_are_clamped():
    cache, _ = fresh(4, 1, 32, 16, "int8")
    x = torch.ones(8, 1, 32, device=DEV)
    cache.write(x, x, ints([[0], [1], [2]]), ints([0, 0, 0]), ints([-3, 4, 2, 2 ** 31 - 1]))
    k, _ = cache.read(ints([[0], [1], [2]]), ints([0, 0, 0]), ints([0, 4, 4, 8]), 8, dtype=torch.float32)
    assert bool((k == 1).all())
    empty = x[:0]
    cache.write(empty, empty, ints([[0]]), ints([0]), ints([0, 0]))
    k, v = cache.read(ints([[0]]), ints([0]), ints([0, 0]), 0)
    assert k.shape == (0, 1, 32) and v.shape == (0, 1, 32)


# ---- attention ----------------------------------------------------------------

ATTENTION_CASES = [  # q heads, kv heads, dim, page, cached lengths, new tokens, causal, window
    (8, 2, 128, 16, [1], [1], True, 0),
    (8, 1, 128, 16, [17, 300, 1, 64], [1, 1, 1, 1], True, 0),
    (4, 4, 64, 32, [33, 0, 500], [1, 0, 1], True, 0),            # a sequence of no tokens
    (32, 2, 128, 64, [700], [1], True, 0),                       # 16 heads a key head
    (40, 2, 64, 16, [130], [1], True, 0),                        # 20: more than one tile of rows
    (6, 3, 80, 16, [40, 7], [5, 7], True, 0),
    (2, 1, 96, 128, [129, 128, 127], [3, 128, 2], True, 0),
    (3, 1, 7, 16, [50], [4], True, 0),
    (2, 2, 1, 16, [20], [20], True, 0),
    (2, 1, 256, 32, [90, 33], [33, 1], True, 0),
    (2, 1, 192, 64, [150], [2], True, 0),
    (4, 2, 128, 16, [200, 90], [70, 90], True, 0),               # prompts, with and without a prefix
    (4, 2, 64, 64, [257], [257], True, 0),
    (4, 2, 128, 32, [150, 40], [150, 40], False, 0),             # no causal mask
    (4, 2, 128, 16, [333, 20], [100, 20], True, 33),             # windows
    (4, 2, 64, 16, [333, 20], [1, 1], True, 16),
    (4, 2, 64, 16, [100], [9], False, 5),
    (4, 2, 64, 16, [5, 3], [9, 3], True, 0),                     # more queries than tokens: rows left with nothing
    (4, 1, 32, 128, [1000], [6], True, 1),
    (1, 1, 160, 64, [222], [130], True, 100),
    (24, 8, 128, 32, [515], [130], True, 0),
]


def build(case, fmt, dtype, seed=0, gain=1.0):
    hq, hk, dim, page, lengths, new, causal, window = case
    g, dt = gen(seed + dim + sum(lengths)), DT[dtype]
    width = max(1, (max(lengths) + page - 1) // page) + 1
    pages = len(lengths) * width + 1
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    table = [order[b * width:(b + 1) * width] for b in range(len(lengths))]
    for b, n in enumerate(lengths):  # what a sequence does not need it does not have
        for i in range((n + page - 1) // page, width):
            table[b][i] = -1
    cache, want = fresh(pages, hk, dim, page, fmt)
    off = offsets_of(lengths)
    k = (torch.randn(off[-1], hk, dim, generator=g, device=DEV) * gain).to(dt)
    v = torch.randn(off[-1], hk, dim, generator=g, device=DEV).to(dt)
    v = v * torch.exp(2 * torch.randn(off[-1], 1, 1, generator=g, device=DEV)).to(dt)  # uneven page scales
    zeros = [0] * len(lengths)
    cache.write(k, v, ints(table), ints(zeros), ints(off))
    want.write(k, v, table, zeros, off)
    # Queries in rows wider than the heads.
    q = torch.randn(sum(new), hq, dim + 8, generator=g, device=DEV).to(dt)[:, :, 5:5 + dim] * 2
    return cache, want, table, q


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("case", ATTENTION_CASES, ids=lambda c: "h%d-%d-d%d-p%d-n%s" % (c[:4] + (sum(c[5]),)))
def test_attention(case, fmt, dtype):
    hq, hk, dim, page, lengths, new, causal, window = case
    say("case attention", case, fmt, dtype)
    cache, want, table, q = build(case, fmt, dtype)
    scale = 1.0 / math.sqrt(dim)
    off = offsets_of(new)
    whole = torch.full((q.shape[0] + 2, hq, dim + 4), 7.0, device=DEV, dtype=q.dtype)
    out = whole[1:-1, :, :dim]
    y = cs.cached_attention(q, cache, ints(table), ints(lengths), ints(off), causal=causal, window=window, out=out)
    exact, mag, smag, top = ref.attention(q, want, table, lengths, off, causal, window, scale)
    within(y, exact, ref.attention_bound(exact, mag, smag, top, dim, q.dtype), "attention %s" % (case,))
    assert bool((whole[0] == 7).all()) and bool((whole[-1] == 7).all()) and bool((whole[..., dim:] == 7).all())


def wide(table, case, work=6e9):
    """The table with room for so many pages (it has none there) that the host, which sees the width alone, plans
    for long sequences: 128-row tiles where a key head has 64 rows, and keys cut into parts."""
    hq, hk, dim, page, lengths, new = case[:6]
    keys = work / (max(1, sum(new) // len(new)) * hq * len(new) * ((dim + 31) // 32 * 32))
    width = max(len(table[0]), min(int(keys) // page + 1, 1 << 20))
    t = torch.full((len(table), width), -1, dtype=torch.int32, device=DEV)
    t[:, :len(table[0])] = ints(table)
    return t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("case", ATTENTION_CASES, ids=lambda c: "h%d-%d-d%d-p%d-n%s" % (c[:4] + (sum(c[5]),)))
def test_attention_planned_for_long_sequences(case, fmt, dtype):
    hq, hk, dim, page, lengths, new, causal, window = case
    say("case attention planned long", case, fmt, dtype)
    cache, want, table, q = build(case, fmt, dtype, seed=2)
    scale = -0.8 / math.sqrt(dim)
    off = offsets_of(new)
    t = wide(table, case)
    tiles = "attention_tiles_kernel" in cs.describe_attention(cache, len(new), sum(new), t.shape[1], hq, DT[dtype], causal, window)
    assert tiles == (sum(new) // len(new) * hq // hk >= 64 and not window), "another kernel than the case is for"
    whole = torch.full((q.shape[0] + 2, hq, dim + 4), 7.0, device=DEV, dtype=q.dtype)
    out = whole[1:-1, :, :dim]
    y = cs.cached_attention(q, cache, t, ints(lengths), ints(off), causal=causal, window=window, scale=scale, out=out)
    exact, mag, smag, top = ref.attention(q, want, table, lengths, off, causal, window, scale)
    within(y, exact, ref.attention_bound(exact, mag, smag, top, dim, q.dtype), "attention %s" % (case,))
    assert bool((whole[0] == 7).all()) and bool((whole[-1] == 7).all()) and bool((whole[..., dim:] == 7).all())


# More of the 128-row kernel: windows, ragged ends, empty rows and idle waves, every width it is built for.
TILE_CASES = [
    (6, 2, 128, 16, [400, 63], [130, 40], True, 90), (8, 1, 64, 64, [500], [33], True, 17),
    (4, 4, 32, 16, [129, 1], [129, 1], True, 0), (4, 2, 96, 32, [65, 190], [100, 190], True, 0),
    (2, 1, 160, 16, [270], [70], False, 0), (2, 1, 192, 128, [260], [90], True, 0), (2, 1, 224, 16, [140], [100], True, 50),
    (2, 1, 256, 64, [300, 90], [64, 64], True, 0), (3, 1, 100, 16, [90], [50], False, 30), (1, 1, 5, 16, [200], [129], True, 0),
    (16, 1, 128, 128, [128], [8], True, 0), (2, 2, 128, 16, [40, 300], [150, 150], True, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("case", TILE_CASES, ids=lambda c: "h%d-%d-d%d-p%d-n%s" % (c[:4] + (sum(c[5]),)))
def test_attention_in_tiles_of_128_rows(case, fmt, dtype):
    hq, hk, dim, page, lengths, new, causal, window = case
    say("case attention tiles", case, fmt, dtype)
    cache, want, table, q = build(case, fmt, dtype, seed=4)
    off, scale = offsets_of(new), 1.0 / math.sqrt(dim)
    exact, mag, smag, top = ref.attention(q, want, table, lengths, off, causal, window, scale)
    # With a window the host plans for no more keys than it leaves: the kernel is reached where many sequences share it.
    n = len(new)
    if window:
        rep = int(6e9 / (sum(new) // n * n * hq * (window + sum(new) // n) * ((dim + 31) // 32 * 32))) + 1
        rep = min(rep, 8192)
    else:
        rep = 1
    t = wide(table, case) if not window else wide(table, case, 0)
    if window and t.shape[1] * page < window + sum(new) // n:
        t = torch.nn.functional.pad(t, (0, (window + sum(new) // n) // page + 1 - t.shape[1]), value=-1)
    assert "attention_tiles_kernel" in cs.describe_attention(cache, n * rep, sum(new) * rep, t.shape[1], hq, DT[dtype], causal, window)
    offs = [0]
    for _ in range(rep):
        offs += [offs[-1] + o for o in off[1:]]
    y = cs.cached_attention(q.repeat(rep, 1, 1), cache, t.repeat(rep, 1), ints(lengths * rep), ints(offs), causal=causal,
                            window=window)
    y = y.view(rep, sum(new), hq, dim)
    within(y[0], exact, ref.attention_bound(exact, mag, smag, top, dim, q.dtype), "tiles %s" % (case,))
    assert bool((y == y[0]).all()), "the same sequence gave two results"


@pytest.mark.parametrize("rows,fmt,dtype", [(128, "int8", "bf16"), (256, "int8", "bf16"), (256, "fp8", "bf16"), (128, "fp8", "f32")])
@pytest.mark.parametrize("dim", [128, 64, 72, 20])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_in_tiles_of_either_height(rows, fmt, dtype, dim, causal):
    """Sequences of unlike lengths in one call, planned for short and for long ones: the tile's height differs, and in
    the higher one waves past the rows, tiles past the keys and blocks past the tokens all occur."""
    case = (4, 1, dim, 16, [400, 63, 200, 17], [130, 40, 200, 20], causal, 0)
    say("case attention heights", rows, fmt, dtype, dim, causal)
    cache, want, table, q = build(case, fmt, dtype, seed=6)
    off, scale = offsets_of(case[5]), 1.0 / math.sqrt(dim)
    exact, mag, smag, top = ref.attention(q, want, table, case[4], off, causal, 0, scale)
    bound = ref.attention_bound(exact, mag, smag, top, dim, q.dtype)
    # High tiles are for 2048 keys and more; below, many sequences have to share the call.
    rep = 1 if rows == 256 or dtype == "f32" else int(2e9 / (sum(case[5]) * 4 * 416 * ((dim + 31) // 32 * 32))) + 1
    t = wide(table, case) if rep == 1 else ints(table)
    t = t.repeat(rep, 1)
    text = cs.describe_attention(cache, 4 * rep, sum(case[5]) * rep, t.shape[1], 4, DT[dtype], causal)
    assert "attention_tiles_kernel" in text and " rows=%d " % rows in text, text
    offs = [0]
    for _ in range(rep):
        offs += [offs[-1] + o for o in off[1:]]
    y = cs.cached_attention(q.repeat(rep, 1, 1), cache, t, ints(case[4] * rep), ints(offs), causal=causal)
    y = y.view(rep, -1, 4, dim)
    within(y[0], exact, bound, "heights")
    assert bool((y == y[0]).all()), "the same sequence gave two results"


@pytest.mark.parametrize("new", [40, 150])
def test_tiles_of_128_rows_ignore_what_lies_behind_masks(new):
    case = (4, 2, 64, 16, [200, 170], [new, new], True, 0)
    cache, want, table, q = build(case, "fp8", "bf16")
    off, lens = ints([0, new, 2 * new]), ints([200, 170])
    t = wide(table, case)
    assert "attention_tiles_kernel" in cs.describe_attention(cache, 2, 2 * new, t.shape[1], 4)
    y = cs.cached_attention(q, cache, t, lens, off)
    k, v = cache.k_codes.view(cache.pages, 2, 16, 64), cache.v_codes.view(cache.pages, 2, 4, 16, 4, 4)
    for bits in (0, 0x7F, 0x80):
        k[table[0][12], :, 8:] = bits
        v[table[0][12], :, 2:] = bits
        assert torch.equal(cs.cached_attention(q, cache, t, lens, off), y)
    # A page in the middle that is not there, a row of NaN, lengths of nothing, and no pages at all.
    hole = t.clone()
    hole[0, 3] = 2 ** 31 - 1
    want.codes["k"] = want.codes["k"].copy()
    rows = [r[:] for r in table]
    rows[0][3] = -1
    exact, mag, smag, top = ref.attention(q, want, rows, [200, 170], [0, new, 2 * new], True, 0, 0.125)
    within(cs.cached_attention(q, cache, hole, lens, off), exact,
           ref.attention_bound(exact, mag, smag, top, 64, q.dtype), "hole")
    bad = q.clone()
    bad[new, 1, 3] = float("nan")
    z = cs.cached_attention(bad, cache, t, lens, off)
    assert bool(z[new, 1].isnan().all())
    clean = y.clone()
    clean[new, 1] = z[new, 1] = 0
    assert torch.equal(z, clean)
    assert bool((cs.cached_attention(q, cache, t, ints([0, -7]), off) == 0).all())
    assert bool((cs.cached_attention(q, cache, torch.full_like(t, -1), lens, off) == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_of_128_rows_with_scales_of_extreme_size(dtype):
    case = (4, 2, 64, 16, [150, 90], [40, 60], True, 0)
    for qgain, scale in ((1.0, 30.0), (1e20, 1e-20), (1e-20, 1e20), (0.0, 1.0), (1.0, 0.0), (3.0, -0.7)):
        cache, want, table, q = build(case, "int8", dtype, seed=5)
        spread = 10.0 ** torch.randint(-20, 21, (cache.pages, 2), device=DEV, generator=gen(9)).float()
        cache.v_scales.mul_(spread)
        want.scales["v"] *= spread.cpu().numpy()
        q = (q.float() * qgain).to(DT[dtype])
        t = wide(table, case)
        assert "attention_tiles_kernel" in cs.describe_attention(cache, 2, 100, t.shape[1], 4, DT[dtype])
        y = cs.cached_attention(q, cache, t, ints([150, 90]), ints([0, 40, 100]), scale=scale)
        exact, mag, smag, top = ref.attention(q, want, table, [150, 90], [0, 40, 100], True, 0, scale)
        within(y, exact, ref.attention_bound(exact, mag, smag, top, 64, q.dtype), "extremes %g %g" % (qgain, scale))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_attention_ignores_what_lies_behind_masks(fmt, new):
    """Pages handed back, rows never written and rows outside the window or
    behind a query have no influence, whatever bits they hold."""
    say("case attention masks", fmt, new)
    case = (4, 2, 64, 16, [200, 170], [new, new], True, 40)
    cache, want, table, q = build(case, fmt, "bf16")
    off = offsets_of([new, new])
    args = (ints([200, 170]), ints(off))
    y = cs.cached_attention(q, cache, ints(table), *args, window=40)
    gone = [row[:] for row in table]
    for b, n in enumerate((200, 170)):
        for i in range(max(0, n - new - 39) // 16):
            gone[b][i] = (-1, 2 ** 31 - 1, -2 ** 31)[i % 3]
    assert torch.equal(cs.cached_attention(q, cache, ints(gone), *args, window=40), y)
    # The rows behind the lengths, in the last pages, and every page of nobody.
    k, v = cache.k_codes.view(cache.pages, 2, 16, 64), cache.v_codes.view(cache.pages, 2, 4, 16, 4, 4)
    for bits in (0, 0x7F, 0x80):
        k[table[0][12], :, 8:] = bits
        v[table[0][12], :, 2:] = bits  # tokens 8.. lie in the third and fourth group of four
        assert torch.equal(cs.cached_attention(q, cache, ints(table), *args, window=40), y)


def test_attention_rows_with_nothing_left_are_zero():
    for new in (1, 20):
        case = (4, 2, 64, 16, [100, 60], [new, new], True, 0)
        cache, want, table, q = build(case, "int8", "bf16")
        none = [[-1] * len(table[0])] * 2
        y = cs.cached_attention(q, cache, ints(none), ints([100, 60]), ints([0, new, 2 * new]))
        assert bool((y == 0).all())
        y = cs.cached_attention(q, cache, ints(table), ints([0, -7]), ints([0, new, 2 * new]))
        assert bool((y == 0).all())
        # No table at all, and no tokens at all.
        y = cs.cached_attention(q, cache, ints([[], []]).view(2, 0), ints([100, 60]), ints([0, new, 2 * new]))
        assert bool((y == 0).all())
        assert cs.cached_attention(q[:0], cache, ints(table), ints([100, 60]), ints([0, 0, 0])).shape[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_scores_far_apart_and_scales_of_extreme_size(dtype):
    """Sharp softmaxes, huge and tiny queries, and values whose pages differ by many
    orders of magnitude: the page of small values may hold the weight."""
    say("case attention extremes", dtype)
    case = (4, 2, 64, 16, [150, 90], [2, 60], True, 0)
    for qgain, scale in ((1.0, 30.0), (1e20, 1e-20), (1e-20, 1e20), (0.0, 1.0), (1.0, 0.0), (3.0, -0.7)):
        cache, want, table, q = build(case, "int8", dtype, seed=5)
        spread = 10.0 ** torch.randint(-20, 21, (cache.pages, 2), device=DEV, generator=gen(9)).float()
        cache.v_scales.mul_(spread)
        want.scales["v"] *= spread.cpu().numpy()
        q = (q.float() * qgain).to(DT[dtype])
        off = offsets_of([2, 60])
        y = cs.cached_attention(q, cache, ints(table), ints([150, 90]), ints(off), scale=scale)
        exact, mag, smag, top = ref.attention(q, want, table, [150, 90], off, True, 0, scale)
        within(y, exact, ref.attention_bound(exact, mag, smag, top, 64, q.dtype),
               "extremes %g %g" % (qgain, scale))


def test_attention_nan_query_spoils_its_own_row_only():
    for new in (1, 40):
        case = (4, 2, 64, 16, [100, 60], [new, new], True, 0)
        cache, want, table, q = build(case, "fp8", "bf16")
        off = ints([0, new, 2 * new])
        clean = cs.cached_attention(q, cache, ints(table), ints([100, 60]), off)
        q = q.clone()
        q[new, 1, 3] = float("nan")
        y = cs.cached_attention(q, cache, ints(table), ints([100, 60]), off)
        assert bool(y[new, 1].isnan().all())
        clean[new, 1] = y[new, 1] = 0
        assert torch.equal(y, clean)


def long_case(length, new, fmt, hq=8, hk=2, dim=128, page=64, seed=1):
    """A long sequence whose reference is computed on the GPU in 64 bits."""
    g = gen(seed)
    pages = (length + page - 1) // page
    order = torch.randperm(pages, generator=g, device=DEV)
    cache = cs.KVCache(pages, hk, dim, page_size=page, fmt=fmt)
    k = torch.randn(length, hk, dim, generator=g, device=DEV).bfloat16()
    v = torch.randn(length, hk, dim, generator=g, device=DEV).bfloat16()
    table = order.to(torch.int32)[None]
    cache.write(k, v, table, ints([0]), ints([0, length]))
    q = torch.randn(new, hq, dim, generator=g, device=DEV).bfloat16()
    k, v = cache.read(table, ints([0]), ints([0, length]), length, dtype=torch.float32)
    k, v = k.double().repeat_interleave(hq // hk, 1), v.double().repeat_interleave(hq // hk, 1)
    exact = torch.empty(new, hq, dim, dtype=torch.float64, device=DEV)
    mag = torch.empty_like(exact)
    for h in range(hq):
        s = q[:, h].double() @ k[:, h].T.contiguous() / math.sqrt(dim)
        p = torch.arange(length - new, length, device=DEV)[:, None]
        s = torch.where(torch.arange(length, device=DEV)[None] <= p, s, torch.full_like(s, -math.inf)).softmax(-1)
        exact[:, h], mag[:, h] = s @ v[:, h], s @ v[:, h].abs()
    return cache, table, q, exact, mag


@pytest.mark.parametrize("length,new,fmt", [(40000, 1, "int8"), (9001, 2, "fp8"), (3000, 700, "int8"), (2047, 2047, "fp8")])
def test_attention_long(length, new, fmt):
    say("case attention long", length, new, fmt)
    cache, table, q, exact, mag = long_case(length, new, fmt)
    y = cs.cached_attention(q, cache, table, ints([length]), ints([0, new]))
    # Scores here have magnitudes' sums under 128 * 4.5 * 4.5 / sqrt(128).
    bound = ref.attention_bound(exact.cpu().numpy(), mag.cpu().numpy(), 230.0, 0.0, 128, torch.bfloat16)
    within(y, exact, bound, "long")
    for _ in range(3):
        assert torch.equal(cs.cached_attention(q, cache, table, ints([length]), ints([0, new])), y)


def test_cache_of_more_than_32_bits_of_bytes():
    """Pages whose codes lie beyond 4 GiB from the start."""
    heads, dim, page = 8, 256, 128
    pages = (1 << 32) // (heads * dim * page) + 40
    cache = cs.KVCache(pages, heads, dim, page_size=page)
    x = torch.randn(page + 9, heads, dim, device=DEV).bfloat16()
    table = ints([[pages - 1, pages - 3]])
    cache.write(x, x, table, ints([0]), ints([0, page + 9]))
    k, v = cache.read(table, ints([0]), ints([0, page + 9]), page + 9)
    # Half a step of the block's scale, and the rounding of the value read to bf16.
    bound = float(x.abs().max()) * (0.5 / 127 + 2.0 ** -8) * 1.01
    assert torch.equal(k, v) and float((k.float() - x.float()).abs().max()) <= bound
    for n in (1, 100):
        q = torch.randn(n, heads, dim, device=DEV).bfloat16()
        y = cs.cached_attention(q, cache, table, ints([page + 9]), ints([0, n]))
        small = cs.KVCache(2, heads, dim, page_size=page)
        small.write(x, x, ints([[0, 1]]), ints([0]), ints([0, page + 9]))
        assert torch.equal(cs.cached_attention(q, small, ints([[0, 1]]), ints([page + 9]), ints([0, n])), y)


# ---- together -------------------------------------------------------------------

def test_calls_run_on_the_current_stream_and_replay_from_a_graph():
    """One generated token through all operators: eagerly, on a side stream, and from a captured graph replayed with
    other inputs, eager work in between."""
    g = gen(3)
    hq, hk, dim, page, width = 8, 2, 64, 16, 256
    wqkv = (torch.randn((hq + 2 * hk) * dim, width, generator=g, device=DEV) / 16).bfloat16()
    wo = (torch.randn(width, hq * dim, generator=g, device=DEV) / 22).bfloat16()
    cos, sin = rope_tables(4096, dim)
    table, off = ints([[3, 1, 0, 2]]), ints([0, 1])
    x, start, length = torch.randn(1, width, generator=g, device=DEV).bfloat16(), ints([0]), ints([1])

    def step(cache):
        qkv = cs.linear(x, wqkv).view(1, hq + 2 * hk, dim)
        q, k = cs.qk_norm_rope(qkv[:, :hq], qkv[:, hq:hq + hk], start, cos, sin)
        cache.write(k, qkv[:, hq + hk:], table, start, off)
        y = cs.cached_attention(q, cache, table, length, off)
        return cs.linear(y.view(1, -1), wo, residual=x)

    inputs = torch.randn(40, 1, width, generator=g, device=DEV).bfloat16()

    def play(run):
        outs = []
        for i in range(40):
            x.copy_(inputs[i])
            start.fill_(i)
            length.fill_(i + 1)
            outs.append(run().clone())
        torch.cuda.synchronize()
        return torch.stack(outs)

    eager = cs.KVCache(4, hk, dim, page_size=page)
    want = play(lambda: step(eager))
    side_cache = cs.KVCache(4, hk, dim, page_size=page)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = play(lambda: step(side_cache))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    cache = cs.KVCache(4, hk, dim, page_size=page)
    start.fill_(0)
    length.fill_(1)
    step(cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step(cache)

    def replay():
        graph.replay()
        (x.float() @ wqkv.float().t()).sum()  # other work in between
        return y

    assert torch.equal(play(replay), want)
