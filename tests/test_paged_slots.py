"""paged.slots on the host (no GPU needed): cache rows of tokens by the table of pages."""

import numpy as np
import pytest

paged = pytest.importorskip("paper_2605_06892_amd.paged")

TABLE = np.array([[3, 0, 7], [5, -1, 2]], dtype=np.int32)


@pytest.mark.parametrize("dtype", [np.int32, np.int64])
def test_rows_of_tokens(dtype):
    seqs, pos = np.array([0, 0, 0, 1, 1, 0], dtype), np.array([0, 15, 16, 3, 47, 33], dtype)
    rows = paged.slots(TABLE, 16, seqs, pos)
    assert rows.dtype == np.int32 and rows.tolist() == [48, 63, 0, 83, 47, 113]
    assert paged.slots(TABLE, 1, [0, 1], [1, 2]).tolist() == [0, 2]
    assert paged.slots(TABLE, 16, seqs[:0], pos[:0]).tolist() == []


def test_tokens_without_a_row():
    """A missing page and a padded position or sequence have no row: -1, which hsa_cache_store skips. They are not the
    row that counting from the end would find."""
    assert paged.slots(TABLE, 16, [1, 1, 0, 0, 0, -1, -9], [16, 31, -1, -16, -999, 4, 4]).tolist() == [-1] * 7


def test_page_numbers_past_the_int32_rows():
    """Page numbers whose rows do not fit int32 belong to no cache, and must not wrap to a row of another page."""
    table = np.array([[2 ** 28, 2 ** 31 - 1, -2 ** 31, 2 ** 27, 2 ** 27 - 1]], dtype=np.int32)
    rows = paged.slots(table, 16, [0] * 6, [5, 16, 32, 48, 64, 79])
    assert rows.tolist() == [-1, -1, -1, -1, 2 ** 31 - 16, 2 ** 31 - 1]


def test_positions_past_the_table():
    with pytest.raises(IndexError):
        paged.slots(TABLE, 16, [0], [48])


@pytest.mark.parametrize("e4m3", [False, True])
def test_layers_may_share_one_workspace(e4m3):
    import torch

    a = paged.PagedCache.allocate(4, 16, 2, 64, torch.float32, device="cpu", e4m3=e4m3)
    b = paged.PagedCache.allocate(4, 16, 2, 64, torch.float32, device="cpu", e4m3=e4m3, workspace=a.workspace)
    assert b.workspace is a.workspace and a.workspace.numel() == paged.H.PAGED_WORKSPACE_BYTES
    assert b.k.data_ptr() != a.k.data_ptr() and b.n_pages == 4
