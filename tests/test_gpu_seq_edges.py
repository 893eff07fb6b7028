"""GPU tests of the calls over several sequences where memory holds what no row wrote, where no score is
finite, and at the limits of fp32. Definitions, bounds and helpers are those of test_gpu_seq.py."""

import math

import pytest
import torch

from paper_2605_06892_amd import hsa_step as H
from test_gpu_seq import _gen, check, form, packed_inputs, packed_want, paged_inputs, paged_want, run_packed, run_paged  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 24, 32, 64])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("exponent", [-128, -127, 127])
def test_paged_exponents_of_rows_that_are_not_there(dtype, page, wide, dh, exponent):
    """e4m3 caches whose exponent bytes were never written but for the sequences' rows, as in memory fresh from the
    allocator: -128 would be 2^-128, which fp32 has not. Rows past a length, in pages outside the cache and in the
    cache's first page, which no sequence names, leave no trace whatever their exponents and codes are."""
    heads, kv, lens = 6, 3, [70, 33, 131, 1]
    q, k, v, held, table = paged_inputs(page + dh, dtype, "e4m3", lens, page, heads, kv, dh,
                                        max_pages=5000 // page if wide else None)
    # a page in front of the others
    k, v = (torch.cat([torch.zeros(page, kv * dh).to(x.dtype), x]) for x in (k, v))
    held = [torch.cat([torch.zeros(page, x.shape[1], dtype=torch.uint8), x.view(torch.uint8)]).view(x.dtype) for x in held]
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
        codes = c.view(torch.uint8)
        codes[~used] = torch.randint(0, 256, codes.shape, generator=_gen(1)).to(torch.uint8)[~used]
    scale = dh ** -0.5
    o, lse = run_paged(q, held, table, lens, page, heads, kv, dh, scale)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, n_pages, heads, kv, dh, scale)
    check(o, lse, want, lw, A, S, dtype, max(lens), dh)


def no_finite_scores(k, q, dh, group):
    """Scores of -infinity for every key and query of the first key/value head: channel 0 is infinite in its keys and
    negative in its queries."""
    k[:, 0] = math.inf
    q[:, :group * dh:dh] = -1.0


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_rows_without_a_finite_score(form, dh, causal):
    """o = 0 and lse = -infinity where every score is -infinity, whatever the values hold: infinities and NaN in blocks
    that every row sees whole and in others. The other key/value head is as ever."""
    dtype, heads, kv, scale = form, 4, 2, dh ** -0.5
    lens_q, lens_k = [5, 700, 40, 30], [5, 700, 300, 7]
    q, k, v, cu_q, cu_k = packed_inputs(41, dtype, lens_q, lens_k, heads, kv, dh)
    no_finite_scores(k, q, dh, heads // kv)
    for at, x in ((2, math.nan), (5 + 3, math.inf), (5 + 350, -math.inf), (5 + 690, math.nan), (705 + 1, math.inf),
                  (705 + 299, math.inf), (1005 + 6, -math.inf)):
        v[at, at % dh] = x
    o, lse = run_packed(q, k, v, cu_q, cu_k, heads, kv, dh, scale, causal)
    half = heads // kv
    assert torch.all(o[:, :half * dh] == 0), o[:, :half * dh].isnan().sum()
    assert torch.all(lse[:, :half] == -math.inf)
    want, lw, A, S = packed_want(q[:, half * dh:], k[:, dh:], v[:, dh:], cu_q, cu_k, half, 1, dh, scale, causal)
    check(o[:, half * dh:], lse[:, half:], want, lw, A, S, dtype, 700, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [24, 64])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_paged_rows_without_a_finite_score(dtype, page, wide, dh):
    heads, kv, lens, scale = 4, 2, [700, 33, 1], dh ** -0.5
    q, k, v, held, table = paged_inputs(42, dtype, dtype, lens, page, heads, kv, dh, max_pages=5000 // page if wide else None)
    no_finite_scores(k, q, dh, heads // kv)
    v[::7, 3], v[::11, 5], v[::13, 9] = math.inf, -math.inf, math.nan
    o, lse = run_paged(q, (k, v, None, None), table, lens, page, heads, kv, dh, scale)
    half = heads // kv
    assert torch.all(o[:, :half * dh] == 0), o[:, :half * dh].isnan().sum()
    assert torch.all(lse[:, :half] == -math.inf)
    want, lw, A, S = paged_want(q[:, half * dh:], k[:, dh:], v[:, dh:], table, lens, page, k.shape[0] // page, half, 1, dh, scale)
    check(o[:, half * dh:], lse[:, half:], want, lw, A, S, dtype, 700, dh)


@pytest.mark.parametrize("page", [24, 64])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("small", ["keys", "queries"])
def test_paged_f32_queries_and_codes_of_very_different_magnitude(dh, page, small):
    """Queries around 2^120 over keys around 2^-110: their products fit fp32, those of queries and codes, without the
    exponents, do not. And 2^-112 over 2^112."""
    heads, kv, lens = 4, 2, [90, 33]
    q, k, v, held, table = paged_inputs(43, "f32", "e4m3", lens, page, heads, kv, dh)
    up, down = (120, -110) if small == "keys" else (-112, 112)
    q = q.clamp(-3, 3) * 2.0 ** up
    held[2].copy_((held[2].long() + down).clamp(-117, 119).to(torch.int8))
    codes = held[0].float().double().view(-1, kv, dh)
    k = (codes * torch.pow(2.0, held[2].double())[..., None]).view(k.shape)
    scale = 2.0 ** -(up + down) * dh ** -0.5
    o, lse = run_paged(q, held, table, lens, page, heads, kv, dh, scale)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, k.shape[0] // page, heads, kv, dh, scale)
    check(o, lse, want, lw, A, S, "f32", 90, dh)


def test_packed_forced_tiles(monkeypatch):
    """HSA_PACKED_TILE: 128 and 256 rows both mean the large kernel, whichever it has for the width; a shape that no
    kernel has is refused; the variable is read at every call."""
    q, k, v, cu, _ = packed_inputs(44, "bf16", [300], [300], 2, 1, 128)
    outs = {}
    for tile in ("16x4", "16x8", "32x4", "128x4", "256x8"):
        monkeypatch.setenv("HSA_PACKED_TILE", tile)
        outs[tile] = run_packed(q, k, v, cu, cu, 2, 1, 128, 0.1, True)[1]
    assert torch.equal(outs["128x4"], outs["256x8"])
    assert not torch.equal(outs["16x4"], outs["256x8"]) and not torch.equal(outs["16x8"], outs["16x4"])
    for tile in ("17x4", "16x5", "128x8", "0x0", "-16x4", "16", "large", "32x4 "):
        monkeypatch.setenv("HSA_PACKED_TILE", tile)
        with pytest.raises(H.HsaStepError if tile in ("17x4", "16x5", "128x8") else ValueError):
            run_packed(q, k, v, cu, cu, 2, 1, 128, 0.1, True)
    monkeypatch.setenv("HSA_PACKED_TILE", "32x4")
    with pytest.raises(H.HsaStepError):  # fp32 has no 32-row tile
        run_packed(q.float(), k.float(), v.float(), cu, cu, 2, 1, 128, 0.1, True)
    monkeypatch.delenv("HSA_PACKED_TILE")
    run_packed(q, k, v, cu, cu, 2, 1, 128, 0.1, True)
