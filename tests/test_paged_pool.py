"""Host side of paged.py's caches in 4 bits and its pool of pages (no GPU needed)."""

import pytest
import torch

paged = pytest.importorskip("paper_2605_06892_amd.paged")


def test_cache_in_4_bits():
    c = paged.PagedCache.allocate(6, 16, 3, 64, torch.bfloat16, device="cpu", e2m1=True)
    assert c.k.dtype == torch.uint8 and tuple(c.k.shape) == (96, 96) and c.k_exp.dtype == torch.int8
    assert tuple(c.v_exp.shape) == (96, 6) and c.n_pages == 6 and c.scale == 0.125
    a = paged.PagedCache.allocate(6, 16, 3, 64, torch.bfloat16, device="cpu", e2m1=True, workspace=c.workspace)
    assert a.workspace is c.workspace
    with pytest.raises(ValueError):
        paged.PagedCache.allocate(6, 16, 3, 64, torch.bfloat16, device="cpu", e4m3=True, e2m1=True)


def test_pages_go_back_to_the_ring():
    p = paged.PagePool.allocate(7, 16, 3, 4, 20, device="cpu")
    assert tuple(p.page_table.shape) == (3, 4) and torch.all(p.page_table == -1) and p.free_at.tolist() == [0, 7, 0]
    # two sequences of 33 and 16 rows, as a plan of theirs leaves the pool: pages 0 to 3 are taken
    p.page_table[0, :3], p.page_table[2, :1] = torch.tensor([0, 1, 2], dtype=torch.int32), 3
    p.lens[:] = torch.tensor([33, 0, 16])
    p.free_at[:] = torch.tensor([4, 3, 0])
    p.release(0)
    assert p.free_at.tolist() == [4, 6, 0] and p.lens.tolist() == [0, 0, 16] and p.free.tolist() == [0, 1, 2, 3, 4, 5, 6]
    p.release(2)
    assert p.free_at.tolist() == [4, 7, 0] and p.free[(4 + torch.arange(7)) % 7].tolist() == [4, 5, 6, 0, 1, 2, 3]
    assert torch.all(p.page_table == -1)
    p.release(1)  # has none
    assert p.free_at.tolist() == [4, 7, 0]
    # a page that was lacking is none to give back
    p.page_table[1, :2], p.lens[1] = torch.tensor([4, -1], dtype=torch.int32), 20
    p.free_at[:] = torch.tensor([5, 6, 1])
    p.release(1)
    assert p.free_at.tolist() == [5, 7, 1] and int(p.free[(5 + 6) % 7]) == 4
