"""GPU tests of rows in 4 bits: caches and weights in e2m1 groups, products with such weights, attention over such
caches, against definitions in 64 bits.

Rows are held to their definition bit for bit. Attention is held to the bounds of test_gpu_seq.py, which do not
depend on how its rows are held. Products, per output element (u = 2^-24, a half step of fp32):
  - a sum of d_in products, which are exact or rounded once with their addition: (d_in + 16) u A with A = sum |x| |w|,
    twice that where the matrix instructions truncate what they align;
  - the row scale: a rounding of the result;
  - GELU: 1.13 times the error of its argument, and of its own value 16 u (1 + |y|), y its argument's polynomial: the
    exponential is as exact as its argument 2 y, which is rounded;
  - the output: half a step of its type.
"""

import math

import numpy as np
import pytest
import torch

import test_gpu_seq as S
from gpu_util import Guarded
from paper_2605_06892_amd import hsa_step as H

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
T = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32
VALUES = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def quantize4(x):
    """Codes' values, the codes and the exponents by the definition, in 64 bits: x [n, d] on the host."""
    y = x.double().view(x.shape[0], -1, GROUP).numpy()
    bad = ~np.isfinite(y).all(-1)
    top = np.where(np.isfinite(y), np.abs(y), 0.0).max(-1)
    e = np.full(top.shape, -125, dtype=np.int64)
    for _ in range(250):
        e = np.where((top > 6.0 * 2.0 ** e.astype(np.float64)) & (e < 125), e + 1, e)
    z = np.where(np.isfinite(y), y, 0.0) * 2.0 ** (-e[..., None].astype(np.float64))
    mag = np.minimum(np.abs(z), 6.0)
    code = np.zeros(z.shape, dtype=np.int64)
    for c in range(1, 8):  # past the middle of two codes, or on it where the upper one is even
        mid = (VALUES[c - 1] + VALUES[c]) / 2
        code = np.where((mag > mid) | ((mag == mid) & (c % 2 == 0)), c, code)
    value = np.copysign(VALUES[code], z) * 2.0 ** e[..., None].astype(np.float64)
    value = np.where(bad[..., None], np.nan, value)
    code = code + 8 * np.signbit(z)
    shape = tuple(x.shape)
    code = code.reshape(shape)
    packed = (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)
    e = np.where(bad, -128, e)
    return torch.from_numpy(value.reshape(shape)), torch.from_numpy(packed), torch.from_numpy(e.astype(np.int8))


def values4(codes, ex):
    """Values of packed codes in 64 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = torch.from_numpy(VALUES)[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    e = ex.double()
    return (v.view(*ex.shape, GROUP) * torch.where(e == -128, math.nan, 2.0 ** e)[..., None]).flatten(-2)


def same_codes(codes, packed, ex):
    """Equal bytes but where the group reads as NaN whatever its codes are."""
    bad = (ex == -128).repeat_interleave(GROUP // 2, -1)
    return bool(torch.all((codes == packed) | bad))


def odd_rows(g, dtype, n, d):
    """Rows of every kind: ordinary, tiny, huge, zero, on the ties, at the limits, not finite."""
    x = S._randn(g, n, d)
    x *= torch.exp(S._randn(g, n, 1) * 20).clamp(1e-38, 1e37)
    x[::7, ::5] *= 100
    i = torch.arange(d)
    ties = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    kinds = [torch.zeros(d), torch.full((d,), 6.0), torch.full((d,), 6.03125), ties[i % 8], -ties[i % 8],
             torch.where(i % 32 == 3, 6.0, i % 32 / 64.0), torch.full((d,), 1e-40), torch.full((d,), 3.3e38),
             -torch.full((d,), 3.38e38), torch.full((d,), 2.0 ** -126), i * 2.0 ** -130, torch.full((d,), 6 * 2.0 ** 125),
             torch.where(i % 67 == 40, math.inf, 1.5), torch.where(i % 71 == 1, math.nan, -2.5), torch.full((d,), -math.inf),
             torch.full((d,), math.nan), torch.where(i % 32 == 31, 1.5 * 2.0 ** 127, 1.0), torch.full((d,), -0.0),
             torch.where(i % 32 == 0, 2.0 ** -125 * 1.5, 2.0 ** -127)]
    for j, row in enumerate(kinds):
        if j < n:
            x[j] = row
    return x.to(T[dtype])


@pytest.mark.parametrize("n,n_rows,kv", [(1, 1, 1), (3, 9, 5), (40, 64, 3), (16, 4096, 8), (777, 1000, 12), (2049, 2049, 2)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_and_load(dtype, dh, n, n_rows, kv):
    g = S._gen(n + dh)
    d = kv * dh
    fused = torch.cat([odd_rows(g, dtype, n, d), S._randn(g, n, d).to(T[dtype])], 1).to(DEV)
    k, v = fused[:, :d], fused[:, d:]
    idx = torch.randperm(n_rows, generator=g)[:n].to(torch.int32)
    if n > 2:
        idx[1], idx[2] = -1, n_rows
    caches = [Guarded((n_rows, d // 2), torch.uint8, s) for s in (1, 2)]
    ex = [Guarded((n_rows, d // GROUP), torch.int8, s) for s in (3, 4)]
    for c, e in zip(caches, ex):
        c.t.fill_(0x5a)
        e.t.fill_(33)
    H.hsa_cache_store(k, v, idx.to(DEV), n, kv, caches[0].t, caches[1].t, ex[0].t, ex[1].t)
    ok = (idx >= 0) & (idx < n_rows)
    rows = idx[ok].long()
    back = [Guarded((n, d), T[dtype], s) for s in (5, 6)]
    H.hsa_cache_load(caches[0].t, caches[1].t, idx.to(DEV), n, kv, back[0].t, back[1].t, ex[0].t, ex[1].t)
    for x, c, e, b in zip((k, v), caches, ex, back):
        value, packed, e_want = quantize4(x.cpu())
        codes, e_got = c.t.cpu(), e.t.cpu()
        assert torch.equal(e_got[rows], e_want[ok]) and same_codes(codes[rows], packed[ok], e_want[ok])
        rest = torch.ones(n_rows, dtype=torch.bool)
        rest[rows] = False
        assert torch.all(codes[rest] == 0x5a) and torch.all(e_got[rest] == 33)
        want = torch.where(ok[:, None], value, torch.zeros_like(value))
        assert S.same(b.t, want)
        for y in (c, e, b):
            y.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_reads_back(dtype):
    """All pairs of codes with every exponent, and a row that is loaded twice."""
    n = 252
    codes = torch.arange(256, dtype=torch.uint8).repeat(n, 1)
    ex = torch.tensor([-128] + list(range(-125, 126)), dtype=torch.int8)[:, None].repeat(1, 512 // GROUP)
    idx = torch.cat([torch.arange(n), torch.tensor([7, 7])]).to(torch.int32)
    c, e = codes.to(DEV), ex.to(DEV)
    out = [torch.empty(n + 2, 512, dtype=T[dtype], device=DEV) for _ in range(2)]
    H.hsa_cache_load(c, c, idx.to(DEV), n + 2, 4, out[0], out[1], e, e)
    want = values4(codes, ex)[idx.long()]
    assert S.same(out[0], want) and S.same(out[1], want)


@pytest.mark.parametrize("n,d,pad", [(1, 32, 0), (3, 64, 8), (17, 96, 0), (257, 1536, 24), (1537, 8960, 0), (5, 4160, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_weights(dtype, n, d, pad):
    w = odd_rows(S._gen(n + d), dtype, n, d + pad).to(DEV)[:, :d]
    codes, ex = Guarded((n, d // 2), torch.uint8, 1), Guarded((n, d // GROUP), torch.int8, 2)
    H.hsa_quantize_w4(w, codes.t, ex.t)
    _, packed, e_want = quantize4(w.cpu())
    assert torch.equal(ex.t.cpu(), e_want) and same_codes(codes.t.cpu(), packed, e_want)
    codes.check()
    ex.check()


# ---------------------------------------------------------------- products


def linear_case(seed, dtype, rows, d_in, d_out):
    g = S._gen(seed)
    x = S._randn(g, rows, d_in)
    x[:, 7::64] *= 8
    codes = torch.randint(0, 256, (d_out, d_in // 2), generator=g).to(torch.uint8)
    ex = torch.randint(-9, 3, (d_out, d_in // GROUP), generator=g).to(torch.int8)
    return x.to(T[dtype]), codes, ex


def linear_check(got, x, codes, ex, out, scale=None, residual=None, gelu=False):
    w, x64 = values4(codes, ex), x.double()
    d_in = x.shape[1]
    z, A = x64 @ w.t(), x64.abs() @ w.abs().t()
    bar = 2 * (d_in + 16) * U * A
    if scale is not None:
        z, bar = z * scale.double()[:, None], bar * scale.double().abs()[:, None]
        bar = bar + 2 * U * z.abs()
    if gelu:
        y = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        z = z * torch.sigmoid(2 * y)
        bar = 1.13 * bar + 16 * U * (1 + y.abs()) * z.abs() + 1e-37
    if residual is not None:
        z = z + residual.double()
        bar = bar + U * z.abs()
    bar = bar + torch.finfo(T[out]).eps / 2 * (z.abs() + bar) + 1e-37
    off = (got.cpu().double() - z).abs()
    assert torch.all(off <= bar), f"{float((off / bar).max()):.2f} of the bound"


LINEAR = [(1, 32, 1), (1, 64, 5), (2, 96, 16), (1, 1536, 1000), (7, 160, 33), (16, 512, 100), (17, 1024, 64), (33, 992, 47),
          (5, 8960, 257), (64, 128, 130), (65, 4128, 31), (130, 256, 17), (3, 16384, 40), (12, 1056, 2050), (1, 4096, 8193)]


@pytest.mark.parametrize("rows,d_in,d_out", LINEAR)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_linear(dtype, out, rows, d_in, d_out):
    x, codes, ex = linear_case(rows + d_in, dtype, rows, d_in, d_out)
    y = Guarded((rows, d_out), T[out], 1)
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t)
    linear_check(y.t, x, codes, ex, out)
    y.check("y")


# every shape of launch: the outputs that ask for 1, 2, 4 and 8 waves beside each other, one and more tiles of rows, splits
# that end inside a unit of 512 inputs, and products shorter than one
SHAPES = [(r, k, n) for n in (200, 4100, 8200) for r, k in ((1, 544), (5, 4640), (16, 1056), (17, 2080), (33, 544), (64, 96))] + \
    [(21, 96, 16400), (11, 608, 16400), (3, 1120, 16400), (32, 608, 32800), (64, 544, 32800), (33, 64, 32800)]


@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_every_launch(dtype, rows, d_in, d_out):
    x, codes, ex = linear_case(rows + d_out, dtype, rows, d_in, d_out)
    y = Guarded((rows, d_out), T[dtype], 1)
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t)
    linear_check(y.t, x, codes, ex, dtype)
    y.check("y")


@pytest.mark.parametrize("units", [2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 13, 16, 18, 25])
@pytest.mark.parametrize("less", [0, 480])
@pytest.mark.parametrize("dtype,rows", [("bf16", 3), ("bf16", 16), ("bf16", 20), ("f32", 1), ("f32", 5), ("f32", 9)])
def test_linear_every_split(dtype, rows, units, less):
    """Few outputs, whose inputs are taken by up to 8 waves in turns: full ones, and some of a last unit of one group."""
    x, codes, ex = linear_case(units, dtype, rows, units * 512 - less, 100)
    y = Guarded((rows, 100), T[dtype], 1)
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t)
    linear_check(y.t, x, codes, ex, dtype)
    y.check("y")


@pytest.mark.parametrize("rows,d_in,d_out", [
    (16, 608, 24600), (20, 1120, 24600), (41, 96, 24600),     # four tiles of five rows, eight waves that share them
    (6, 4640, 19700), (10, 608, 24600), (33, 544, 9900),      # two tiles, eight waves
    (7, 4128, 9900), (10, 4640, 9900), (10, 544, 9900), (64, 1056, 4900),   # two tiles, four waves, their inputs split or not
    (1, 544, 32800), (5, 1120, 32800), (5, 544, 8200), (8, 4640, 4200), (9, 544, 4200)])  # one tile
def test_linear_every_f32_launch(rows, d_in, d_out):
    x, codes, ex = linear_case(rows + d_out, "f32", rows, d_in, d_out)
    y = Guarded((rows, d_out), torch.float32, 1)
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t)
    linear_check(y.t, x, codes, ex, "f32")
    y.check("y")


@pytest.mark.parametrize("rows,d_in,d_out", [
    (17, 544, 9900), (32, 1056, 9900), (33, 1120, 5300), (64, 4640, 5300),   # two tiles, four waves, their inputs split
    (33, 480, 5300), (128, 544, 5300), (17, 4640, 4200), (40, 4640, 4200),   # one tile, four waves
    (5, 4640, 10300), (16, 4128, 10300), (16, 1056, 8200), (16, 4640, 8200), (3, 4640, 8200), (1, 96, 8200)])
def test_linear_every_bf16_launch(rows, d_in, d_out):
    x, codes, ex = linear_case(rows + d_out, "bf16", rows, d_in, d_out)
    y = Guarded((rows, d_out), torch.bfloat16, 1)
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t)
    linear_check(y.t, x, codes, ex, "bf16")
    y.check("y")


@pytest.mark.parametrize("scale", [-100, -115, -126])
def test_linear_small_f32_rows(scale):
    """fp32 rows are taken to within 2^-133 of each value: with values about 2^-115 that shows in an output of ordinary size."""
    g = S._gen(8)
    x = S._randn(g, 3, 640) * 2.0 ** scale
    codes = torch.randint(0, 256, (70, 320), generator=g).to(torch.uint8)
    ex = torch.randint(100, 111, (70, 20), generator=g).to(torch.int8)
    y = torch.empty(3, 70, device=DEV)
    H.hsa_linear_w4(x.to(DEV), 3, codes.to(DEV), ex.to(DEV), y)
    w = values4(codes, ex)
    want, A = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    bar = 2 * (640 + 16) * U * A + 2.0 ** -133 * w.abs().sum(1) + 1e-37
    off = (y.cpu().double() - want).abs()
    assert torch.all(off <= bar), f"{float((off / bar).max()):.2f} of the bound"


@pytest.mark.parametrize("rows,d_in,d_out", [(1, 64, 7), (9, 1056, 130), (40, 288, 65), (2, 2048, 600)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["scale", "gelu", "scale+gelu", "residual", "scale+residual", "in place", "scale f32"])
def test_linear_epilogues(dtype, what, rows, d_in, d_out):
    g = S._gen(3)
    x, codes, ex = linear_case(rows + d_out, dtype, rows, d_in, d_out)
    out = "f32" if "f32" in what else dtype
    scale = torch.rand(rows, generator=g) + 0.01 if "scale" in what else None
    residual = S._randn(g, rows, d_out).to(T[out]) * 3 if "residual" in what or what == "in place" else None
    y = Guarded((rows, d_out), T[out], 1)
    r = None if residual is None else residual.to(DEV)
    if what == "in place":
        y.t.copy_(r)
        r = y.t
    H.hsa_linear_w4(x.to(DEV), rows, codes.to(DEV), ex.to(DEV), y.t, residual=r,
                    row_scale=None if scale is None else scale.to(DEV), gelu="gelu" in what)
    linear_check(y.t, x, codes, ex, out, scale, residual, "gelu" in what)
    y.check("y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_exact_sums_and_limits(dtype):
    """Small whole numbers: exact. Exponents at their limits; a NaN group and infinite rows stay in their outputs."""
    g = S._gen(1)
    x = torch.randint(-4, 5, (6, 640), generator=g).to(T[dtype])
    codes = torch.randint(0, 256, (50, 320), generator=g).to(torch.uint8)
    ex = torch.full((50, 20), 1, dtype=torch.int8)
    y = torch.empty(6, 50, device=DEV)
    H.hsa_linear_w4(x.to(DEV), 6, codes.to(DEV), ex.to(DEV), y)
    assert torch.equal(y.cpu().double(), x.double() @ values4(codes, ex).t())
    ex[3], ex[4], ex[5, 7] = 125, -125, -128
    codes[3] = 0x02  # a one in every even place: 320 * 0.25 * 2^125 = 3.4e39, past fp32's greatest value
    x = torch.ones_like(x) * 0.25
    x[2, 100] = math.inf
    x[4, 639] = math.nan
    H.hsa_linear_w4(x.to(DEV), 6, codes.to(DEV), ex.to(DEV), y)
    z = y.cpu()
    assert torch.isnan(z[:, 5]).all() and torch.isnan(z[4]).all()
    assert not torch.isfinite(z[2]).any()
    keep = [0, 1, 3, 5]
    want = x[keep].double() @ values4(codes, ex)[[0, 3, 4, 49]].t()
    assert S.same(z[keep][:, [0, 3, 4, 49]], want.float())


def test_linear_rows_of_zeros_and_rows_not_asked_for():
    x, codes, ex = linear_case(1, "bf16", 5, 256, 70)
    y = torch.full((5, 70), 7.0, dtype=torch.bfloat16, device=DEV)
    H.hsa_linear_w4(x.to(DEV), 0, codes.to(DEV), ex.to(DEV), y)
    assert torch.all(y == 7)
    H.hsa_linear_w4(x.to(DEV), 3, codes.to(DEV), ex.to(DEV), y)
    linear_check(y[:3], x[:3], codes, ex, "bf16")
    assert torch.all(y[3:] == 7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_row_by_row(dtype):
    """A row's result is the same bits alone and among others of its tile, and in every run."""
    x, codes, ex = linear_case(2, dtype, 16, 2080, 300)
    x, codes, ex = x.to(DEV), codes.to(DEV), ex.to(DEV)
    y, z = (torch.empty(16, 300, dtype=x.dtype, device=DEV) for _ in range(2))
    H.hsa_linear_w4(x, 16, codes, ex, y)
    for _ in range(3):
        H.hsa_linear_w4(x, 16, codes, ex, z)
        assert torch.equal(y, z)


@pytest.mark.parametrize("dtype,most", [("bf16", 16), ("f32", 5)])
@pytest.mark.parametrize("d_in,d_out", [(2080, 300), (8960, 1537), (512, 17), (5120, 4128), (1536, 8960), (3168, 12288),
                                        (2048, 32784)])  # tiles of outputs from two to eight times the CUs
def test_linear_row_alone_and_among_others(dtype, most, d_in, d_out):
    """Up to 16 bf16 or 5 fp32 rows the inputs are split by d_in and d_out alone, so a row's sums are taken in one order and
    their bits are the same whatever stands beside it. (Larger calls may split otherwise.)"""
    x, codes, ex = linear_case(d_in + d_out, dtype, most, d_in, d_out)
    scale = torch.rand(most, generator=S._gen(1)).to(DEV)
    x, codes, ex = x.to(DEV), codes.to(DEV), ex.to(DEV)
    y = torch.empty(most, d_out, dtype=x.dtype, device=DEV)
    H.hsa_linear_w4(x, most, codes, ex, y, row_scale=scale)
    for first, n in [(i, 1) for i in range(most)] + [(0, 2), (1, 3), (most - 4, 4), (1, most - 1)]:
        z = torch.empty(n, d_out, dtype=x.dtype, device=DEV)
        H.hsa_linear_w4(x[first:first + n], n, codes, ex, z, row_scale=scale[first:first + n])
        assert torch.equal(z, y[first:first + n]), (first, n)


@pytest.mark.parametrize("d_in,d_out", [(16384, 270000)])
def test_linear_offsets_past_32_bits(d_in, d_out):
    """Weights of more than 2^31 bytes: outputs at both ends and in the middle."""
    w = torch.randint(0, 256, (1000, d_in // 2), generator=S._gen(4)).to(torch.uint8)
    codes = w.to(DEV).repeat(d_out // 1000, 1)
    ex = torch.zeros(d_out, d_in // GROUP, dtype=torch.int8, device=DEV)
    x, _, _ = linear_case(5, "bf16", 2, d_in, 1)
    y = torch.empty(2, d_out, device=DEV)
    H.hsa_linear_w4(x.to(DEV), 2, codes, ex, y)
    linear_check(y[:, -1000:], x, w, ex[:1000].cpu(), "f32")
    assert torch.equal(y.view(2, -1, 1000), y[:, :1000][:, None].expand(2, d_out // 1000, 1000))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_as_many_rows_as_it_takes(dtype):
    """2^18 rows: the tiles of rows fit the launch. All rows the same but for a factor that is exact."""
    x, codes, ex = linear_case(9, dtype, 4, 32, 3)
    n = 2 ** 18
    rows = x.to(DEV).repeat(n // 4, 1)
    rows[n // 2:] *= 4
    y = torch.empty(n, 3, dtype=T[dtype], device=DEV)
    H.hsa_linear_w4(rows, n, codes.to(DEV), ex.to(DEV), y)
    linear_check(y[:4], x, codes, ex, dtype)
    assert torch.equal(y[:n // 2].view(-1, 4, 3), y[:4].expand(n // 8, 4, 3)) and torch.equal(y[n // 2:], 4 * y[:n // 2])


def test_linear_other_stream_and_graph():
    x, codes, ex = (t.to(DEV) for t in linear_case(6, "bf16", 3, 1024, 500))
    want, y = (torch.empty(3, 500, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    H.hsa_linear_w4(x, 3, codes, ex, y, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        H.hsa_linear_w4(x, 3, codes, ex, y)
    for i in range(3):
        x.copy_(S._randn(S._gen(i), 3, 1024))
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        H.hsa_linear_w4(x, 3, codes, ex, want)
        assert torch.equal(y, want)


def test_refusals_of_the_binding():
    x, codes, ex = (t.to(DEV) for t in linear_case(6, "bf16", 4, 256, 64))
    y = torch.empty(4, 64, dtype=torch.bfloat16, device=DEV)
    ok = dict(x=x, n_rows=4, w=codes, w_exp=ex, y=y)
    H.hsa_linear_w4(**ok)
    for change in (dict(n_rows=5), dict(w=codes[:, :64].contiguous()), dict(y=y[:, :32].contiguous()), dict(y=y[:3]),
                   dict(residual=y[:2]), dict(row_scale=torch.ones(3, device=DEV)), dict(x=x.t()), dict(w=codes.cpu()),
                   dict(x=x[:, ::2])):
        with pytest.raises(ValueError):
            H.hsa_linear_w4(**{**ok, **change})
    for change in (dict(w=codes.to(torch.int8)), dict(w_exp=ex[:4]), dict(w_exp=ex.int()), dict(x=x.half()), dict(y=y.half()),
                   dict(residual=y.float()), dict(row_scale=torch.ones(4, device=DEV).bfloat16())):
        with pytest.raises(TypeError):
            H.hsa_linear_w4(**{**ok, **change})
    for change in (dict(gelu=True, residual=y.clone()), dict(gelu=True, y=y.float()), dict(x=x.float()), dict(n_rows=-1)):
        with pytest.raises(H.HsaStepError):
            H.hsa_linear_w4(**{**ok, **change})
    w = torch.zeros(8, 256, device=DEV)
    c, e = torch.empty(8, 128, dtype=torch.uint8, device=DEV), torch.empty(8, 8, dtype=torch.int8, device=DEV)
    H.hsa_quantize_w4(w, c, e)
    for a in ((w[:, :250], c, e), (w, c[:4], e), (w.t(), c, e)):
        with pytest.raises(ValueError):
            H.hsa_quantize_w4(*a)
    for a in ((w.half(), c, e), (w, e, e), (w, c, e[:, :4].contiguous()), (w, c, c)):
        with pytest.raises(TypeError):
            H.hsa_quantize_w4(*a)
    k = torch.zeros(8, 256, dtype=torch.bfloat16, device=DEV)
    i = torch.arange(8, dtype=torch.int32, device=DEV)
    ok = dict(k=k, v=k, idx=i, n=8, kv_heads=2, k_cache=c, v_cache=c.clone(), k_exp=e, v_exp=e.clone())
    H.hsa_cache_store(**ok)
    for change in (dict(k_exp=None), dict(v_exp=e[:, :2].contiguous()), dict(v_exp=e[:4])):
        with pytest.raises(TypeError):
            H.hsa_cache_store(**{**ok, **change})
    with pytest.raises(ValueError):
        H.hsa_cache_store(**{**ok, "k": k[:, :128], "v": k[:, :128]})
    with pytest.raises(H.HsaStepError):
        H.hsa_cache_store(**{**ok, "v_cache": c})


# ---------------------------------------------------------------- attention


def paged_inputs4(seed, dtype, lens, page, heads, kv, dh, spare=2, max_pages=None):
    q, k, v, _, table = S.paged_inputs(seed, dtype, dtype, lens, page, heads, kv, dh, spare, max_pages)
    k[:, 5::32] *= 6
    (kv_, kc, ke), (vv, vc, ve) = quantize4(k), quantize4(v)
    return q, kv_, vv, (kc, vc, ke, ve), table


@pytest.mark.parametrize("lens,page,heads,kv", S.PAGED, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged(dtype, wide, dh, lens, page, heads, kv):
    """wide: page tables of 5000 rows, whose launch deals tiles of rows to the workgroups and joins the parts."""
    q, k, v, held, table = paged_inputs4(sum(lens) + page, dtype, lens, page, heads, kv, dh,
                                         max_pages=5000 // page if wide else None)
    o = Guarded(q.shape, T[dtype], 1)
    nb = H.hsa_paged_attention_workspace_bytes(T[dtype], len(lens), heads, kv, dh, table.shape[1] * page)
    ws = Guarded((max(nb, 1),), torch.uint8, 2)
    ws.t.fill_(255)
    _, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, dh ** -0.5, o.t, ws.t)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, kv, dh, dh ** -0.5)
    S.check(o.t, lse, want, lw, A, Sm, dtype, max(lens), dh)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,page,heads,kv,rows", [
    ([900, 70, 0, 1], 32, 140, 140, 2112),      # more items than runs go round: the tiles of all in one order
    ([300, 3], 16, 300, 300, 2064),
    ([3000, 70, 1111], 64, 68, 4, 4096),        # groups of 17: two items of one head beside each other
    ([3000, 70, 1111], 20, 34, 2, 4000),
    ([5000], 64, 24, 8, 8192),
    ([4097, 4096], 32, 6, 6, 4128),
    ([9, 300, 700, 1, 0] * 32, 32, 16, 8, 704),   # short ones, four items to a workgroup
    ([9, 300, 700, 1, 0] * 32, 20, 34, 2, 760),
    ([33, 64, 500] * 60, 64, 6, 6, 512),
], ids=range(9))
def test_paged_every_launch(dtype, lens, page, heads, kv, rows):
    dh = 64
    q, k, v, held, table = paged_inputs4(len(lens), dtype, lens, page, heads, kv, dh, max_pages=rows // page)
    nb = H.hsa_paged_attention_workspace_bytes(T[dtype], len(lens), heads, kv, dh, table.shape[1] * page)
    o, ws = Guarded(q.shape, T[dtype], 1), Guarded((max(nb, 1),), torch.uint8, 2)
    ws.t.fill_(255)
    _, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, 0.125, o.t, ws.t)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, kv, dh, 0.125)
    S.check(o.t, lse, want, lw, A, Sm, dtype, max(lens), dh)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", ["e2m1", "e4m3", "own"])
@pytest.mark.parametrize("heads", [1, 20])
@pytest.mark.parametrize("lens", [[300, 40000, 250, 500], [0, 40000, 1], [257] * 4, [20000, 20001, 0, 0]], ids=range(4))
def test_paged_few_items_of_many_runs(dtype, cache, heads, lens):
    """Outputs joined eight runs to a workgroup, where several of the eight begin an item and where none does."""
    dh, page = 64, 64
    if cache == "e2m1":
        q, k, v, held, table = paged_inputs4(11, dtype, lens, page, heads, 1, dh, max_pages=640)
    else:
        q, k, v, held, table = S.paged_inputs(11, dtype, dtype if cache == "own" else cache, lens, page, heads, 1, dh, max_pages=640)
    nb = H.hsa_paged_attention_workspace_bytes(T[dtype], len(lens), heads, 1, dh, table.shape[1] * page)
    o, ws = Guarded(q.shape, T[dtype], 1), Guarded((nb,), torch.uint8, 2)
    ws.t.fill_(255)
    _, lse = S.run_paged(q, held, table, lens, page, heads, 1, dh, 0.125, o.t, ws.t)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, 1, dh, 0.125)
    S.check(o.t, lse, want, lw, A, Sm, dtype, max(lens), dh)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", ["e2m1", "e4m3", "own"])
@pytest.mark.parametrize("lens,group,kv", [
    ([200] * 16, 16, 1), ([200, 199], 5, 8),   # all begin in the first runs, which have a tile each
    ([1, 0, 129, 128, 127, 4000], 4, 2),
    ([3000 + 131 * i for i in range(16)], 2, 1),  # a little further apart each
    ([40960], 20, 1), ([130], 1, 1)], ids=range(6))
def test_paged_short_sequences_in_wide_tables(dtype, cache, lens, group, kv):
    """Joins of items that begin wherever short sequences leave them in a table of many runs."""
    dh, page, heads = 64, 64, group * kv
    make = S.paged_inputs if cache != "e2m1" else lambda g, d, c, *a, **k: paged_inputs4(g, d, *a, **k)
    q, k, v, held, table = make(len(lens), dtype, dtype if cache == "own" else cache, lens, page, heads, kv, dh, max_pages=640)
    nb = H.hsa_paged_attention_workspace_bytes(T[dtype], len(lens), heads, kv, dh, table.shape[1] * page)
    o, ws = Guarded(q.shape, T[dtype], 1), Guarded((nb,), torch.uint8, 2)
    ws.t.fill_(255)
    _, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, 0.125, o.t, ws.t)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, kv, dh, 0.125)
    S.check(o.t, lse, want, lw, A, Sm, dtype, max(lens), dh)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_pages", [0, 3, 300])
def test_paged_without_rows(dtype, max_pages):
    """No pages in the table, and no pages in the cache: outputs of zeros."""
    q = torch.ones(2, 256, dtype=T[dtype])
    c, e = torch.empty(0, 64, dtype=torch.uint8), torch.empty(0, 4, dtype=torch.int8)
    table = torch.zeros(2, max_pages, dtype=torch.int32)
    o, lse = S.run_paged(q, (c, c, e, e), table, [5, 0], 16, 2, 1, 128, 0.1)
    assert torch.all(o == 0) and torch.all(lse == -math.inf)


@pytest.mark.parametrize("page", [32, 24])
def test_paged_length_at_the_limit(page):
    """The longest length the call takes, all its pages the same two; its waves add up 2^19 weights in each lane at most."""
    q, k, v, held, table = paged_inputs4(31, "bf16", [2 * page], page, 2, 1, 64, spare=0)
    pages = 2 ** 30 // page
    n = pages * page
    table = torch.full((1, pages), int(table[0, 1]), dtype=torch.int32).index_fill(1, torch.tensor([0]), int(table[0, 0]))
    o, lse = S.run_paged(q, held, table, [n], page, 2, 1, 64, 0.125)
    first, rest = int(table[0, 0]) * page, int(table[0, 1]) * page
    for h in range(2):
        s = [(k[r:r + page].double() @ q[0, h * 64:h * 64 + 64].double()) * 0.125 for r in (first, rest)]
        w = torch.cat([s[0], s[1] + math.log(pages - 1)])
        want = torch.softmax(w, 0) @ torch.cat([v[first:first + page], v[rest:rest + page]]).double()
        assert float((o[0, h * 64:h * 64 + 64].cpu().double() - want).abs().max()) < (2.0 ** -7 + 2 ** 20 * U) * float(v.abs().max())
        assert abs(float(lse[0, h]) - float(torch.logsumexp(w, 0))) < 2 ** 19 * U + 1e-5


def test_paged_f32_large_scores():
    """Scores of some thousands in fp32, where one that is off by bf16's step would choose other rows."""
    q, k, v, held, table = paged_inputs4(3, "f32", [300, 77], 16, 4, 2, 64)
    q = q * 300
    o, lse = S.run_paged(q, held, table, [300, 77], 16, 4, 2, 64, 0.125)
    want, lw, A, Sm = S.paged_want(q, k, v, table, [300, 77], 16, k.shape[0] // 16, 4, 2, 64, 0.125)
    S.check(o, lse, want, lw, A, Sm, "f32", 300, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("dh", [64, 128])
def test_paged_many_sequences_and_one_long(dtype, page, dh):
    lens = [(i * 37) % 200 for i in range(150)] + [9000]
    q, k, v, held, table = paged_inputs4(4, dtype, lens, page, 4, 2, dh)
    o, lse = S.run_paged(q, held, table, lens, page, 4, 2, dh, 0.125)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, 4, 2, dh, 0.125)
    S.check(o, lse, want, lw, A, Sm, dtype, 9000, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 24, 32, 64])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("exponent", [-128, -127, 127])
def test_paged_rows_that_are_not_there(dtype, page, wide, dh, exponent):
    """Codes and exponents that were never written, pages outside the cache, and a first page that no sequence names
    leave no trace."""
    heads, kv, lens = 6, 3, [70, 33, 131, 1]
    q, k, v, held, table = paged_inputs4(page + dh, dtype, lens, page, heads, kv, dh,
                                         max_pages=5000 // page if wide else None)
    k, v, *held = (torch.cat([torch.zeros(page, x.shape[1], dtype=x.dtype), x]) for x in (k, v, *held))
    table = torch.where(table >= 0, table + 1, table)
    n_pages = k.shape[0] // page
    if page < 64:
        table[0, 1], table[2, 0], table[2, 2] = -1, n_pages, 2 ** 31 - 1
    used = torch.zeros(n_pages * page, dtype=torch.bool)
    for s, n in enumerate(lens):
        t = torch.arange(n)
        pages = table[s].long()[t // page]
        ok = (pages >= 0) & (pages < n_pages)
        used[(pages * page + t % page)[ok]] = True
    assert not used[:page].any()
    for e in held[2:]:
        e[~used] = exponent
    for c in held[:2]:
        c[~used] = torch.randint(0, 256, c.shape, generator=S._gen(1)).to(torch.uint8)[~used]
    o, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, dh ** -0.5)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, n_pages, heads, kv, dh, dh ** -0.5)
    S.check(o, lse, want, lw, A, Sm, dtype, max(lens), dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_paged_groups_that_are_seen_and_not_finite(dtype, dh, wide):
    """A NaN group of values is 32 NaN channels of the heads that see it, one of keys everything they have."""
    lens, page, heads, kv = [200, 40], 16, 4, 2
    q, k, v, held, table = paged_inputs4(7, dtype, lens, page, heads, kv, dh, max_pages=100 if wide else None)
    want, lw, A, Sm = S.paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, kv, dh, 0.125)
    r = int(table[0, 5]) * page + 3
    held[3][r, 1] = -128  # channels 32 to 63 of the first head's values
    o, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, 0.125)
    nan = torch.zeros(2, heads * dh, dtype=torch.bool)
    for h in range(2):
        nan[0, h * dh + 32:h * dh + 64] = True
    got = o.cpu()
    assert torch.equal(torch.isnan(got), nan)
    S.check(torch.where(nan, torch.zeros_like(got), got), lse, torch.where(nan, 0.0, want), lw, A, Sm, dtype, 200, dh)
    held[2][r, 0] = -128
    o, lse = S.run_paged(q, held, table, lens, page, heads, kv, dh, 0.125)
    assert torch.isnan(o[0, :2 * dh]).all() and torch.isnan(lse[0, :2]).all()
    assert torch.isfinite(o[0, 2 * dh:]).all() and torch.isfinite(o[1]).all() and torch.isfinite(lse[1]).all()


def test_offsets_past_32_bits():
    """Rows whose offset in the cache passes 2^31 bytes: written, read back and attended to."""
    kv, dh, page = 16, 128, 32
    n_pages = 2 ** 31 // (kv * dh // 2 * page) + 40
    n_rows = n_pages * page
    kc, vc = (torch.empty(n_rows, kv * dh // 2, dtype=torch.uint8, device=DEV) for _ in range(2))
    ke, ve = (torch.empty(n_rows, kv * dh // GROUP, dtype=torch.int8, device=DEV) for _ in range(2))
    g = S._gen(1)
    k, v = S._randn(g, 70, kv * dh).bfloat16(), S._randn(g, 70, kv * dh).bfloat16()
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32)
    t = torch.arange(70)
    idx = (table[0].long()[t // page] * page + t % page).to(torch.int32).to(DEV)
    H.hsa_cache_store(k.to(DEV), v.to(DEV), idx, 70, kv, kc, vc, ke, ve)
    kb, vb = (torch.empty(70, kv * dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    H.hsa_cache_load(kc, vc, idx, 70, kv, kb, vb, ke, ve)
    assert S.same(kb, quantize4(k)[0]) and S.same(vb, quantize4(v)[0])
    q = S._randn(g, 1, 2 * kv * dh).bfloat16()
    o = torch.empty(1, 2 * kv * dh, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(H.PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    H.hsa_paged_attention(q.to(DEV), kc, vc, table.to(DEV), torch.tensor([70], dtype=torch.int32, device=DEV), page, 2 * kv, kv,
                          dh, 0.09, o, ws, k_exp=ke, v_exp=ve)
    want, A = torch.zeros(1, 2 * kv * dh).double(), torch.zeros(1, 2 * kv * dh).double()
    for h in range(2 * kv):
        c, ck = slice(h * dh, h * dh + dh), slice(h // 2 * dh, h // 2 * dh + dh)
        want[:, c], _, A[:, c], Sm = S.attend64(q[:, c], kb.cpu()[:, ck], vb.cpu()[:, ck], torch.ones(1, 70, dtype=torch.bool), 0.09)
    S.check(o, None, want, None, A, Sm, "bf16", 70, dh)
