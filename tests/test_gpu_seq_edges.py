"""GPU tests of the calls over several sequences where memory holds what no row wrote. Definitions, bounds
and helpers are those of test_gpu_seq.py."""

import pytest
import torch

from test_gpu_seq import _gen, check, paged_inputs, paged_want, run_paged

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
