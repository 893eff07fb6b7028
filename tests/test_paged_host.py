"""Host side of paged.py's layer with weights in 4 bits: steps that do not fit its buffers are refused before anything is
enqueued (no GPU needed)."""

import pytest
import torch

H = pytest.importorskip("paper_2605_06892_amd.hsa_step")
paged = pytest.importorskip("paper_2605_06892_amd.paged")

D, HEADS, KV, DH = 64, 2, 1, 64


@pytest.fixture
def calls(monkeypatch):
    """The names of the entry points called, none of which does anything."""
    seen = []
    for name in ("hsa_row_rms_scale", "hsa_linear_w4", "hsa_qk_norm_rope", "hsa_packed_attention", "hsa_cache_store",
                 "hsa_paged_attention", "hsa_quantize_w4"):
        monkeypatch.setattr(H, name, lambda *a, _name=name, **k: seen.append(_name))
    return seen


def world(n_tokens, n_seqs, pool_tokens):
    w = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    lay = paged.Layer4.allocate(w((HEADS + 2 * KV) * DH, D), w(D, HEADS * DH), HEADS, KV, DH, n_tokens)
    c = paged.PagedCache.allocate(8, 16, KV, DH, torch.bfloat16, device="cpu", e2m1=True)
    return lay, c, paged.PagePool.allocate(8, 16, n_seqs, 4, pool_tokens, device="cpu")


@pytest.mark.parametrize("n_tokens,n_seqs,pool_tokens,n,prompts", [
    (4, 5, 8, 5, False), (4, 2, 8, 5, True),   # more than the layer has rows
    (8, 5, 4, 5, False), (8, 2, 4, 5, True),   # more than the pool plans
    (8, 3, 8, 4, False), (8, 3, 8, 2, False),  # not one for every sequence
    (8, 3, 8, 0, False)])
def test_step_refuses_what_does_not_fit(calls, n_tokens, n_seqs, pool_tokens, n, prompts):
    lay, c, pool = world(n_tokens, n_seqs, pool_tokens)
    calls.clear()
    x = torch.zeros(n, D, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lay.step(x, c, pool, None, torch.empty_like(x), prompts=prompts)
    assert not calls


def test_step_refuses_an_output_of_other_rows(calls):
    lay, c, pool = world(4, 3, 4)
    calls.clear()
    with pytest.raises(ValueError):
        lay.step(torch.zeros(3, D, dtype=torch.bfloat16), c, pool, None, torch.zeros(4, D, dtype=torch.bfloat16))
    assert not calls


@pytest.mark.parametrize("n_tokens,n_seqs,n,prompts", [(4, 4, 4, False), (4, 2, 4, True), (4, 2, 1, True), (9, 3, 3, False)])
def test_step_takes_what_fits(calls, n_tokens, n_seqs, n, prompts):
    lay, c, pool = world(n_tokens, n_seqs, n_tokens)
    calls.clear()
    x = torch.zeros(n, D, dtype=torch.bfloat16)
    lay.step(x, c, pool, None, x, prompts=prompts)
    assert calls == ["hsa_row_rms_scale", "hsa_linear_w4", "hsa_qk_norm_rope",
                     *(("hsa_packed_attention", "hsa_cache_store") if prompts else ("hsa_cache_store", "hsa_paged_attention")),
                     "hsa_linear_w4"]


@pytest.mark.parametrize("rows,scales,n", [(5, 4, 5), (4, 5, 5), (4, 4, 5)])
def test_row_scales_are_as_many_as_rows(monkeypatch, rows, scales, n):
    """hsa_row_rms_scale knows its tensors' sizes: no kernel is asked to write past them."""
    class Library:
        def hsa_row_rms_scale(self, *a):
            raise AssertionError("enqueued")
    monkeypatch.setattr(H, "_dev", lambda *t: None)
    monkeypatch.setattr(H, "lib", Library)
    with pytest.raises(ValueError):
        H.hsa_row_rms_scale(torch.zeros(rows, 8), n, torch.zeros(scales))


def test_a_sequence_resumes_before_the_page_that_was_lacking():
    p = paged.PagePool.allocate(8, 16, 3, 5, 20, device="cpu")
    # 70 rows whose second page was lacking and whose later pages were not, 20 rows that have theirs, none
    p.page_table[0] = torch.tensor([6, -1, 2, 7, -1], dtype=torch.int32)
    p.page_table[1, :2] = torch.tensor([0, 1], dtype=torch.int32)
    p.lens[:] = torch.tensor([70, 20, 0])
    p.free[:] = torch.tensor([3, 4, 5, 0, 0, 0, 0, 0])
    p.free_at[:] = torch.tensor([0, 3, 2])
    p.lacked[:] = 2
    assert p.resume(1) == 0 and p.resume(2) == 0 and p.lens.tolist() == [70, 20, 0] and p.free_at.tolist() == [0, 3, 2]
    assert p.resume(0) == 54  # rows 16 to 69
    assert p.lens.tolist() == [16, 20, 0] and p.page_table[0].tolist() == [6, -1, -1, -1, -1]
    assert p.free_at.tolist() == [0, 5, 2] and p.free[:5].tolist() == [3, 4, 5, 2, 7]
    assert p.resume(0) == 0 and p.lacked.tolist() == [2]
    p.page_table[1, :2], p.lens[1] = torch.tensor([-1, 1], dtype=torch.int32), 17  # from its first page on
    assert p.resume(1) == 17 and p.lens[1] == 0 and p.free_at.tolist() == [0, 6, 2] and int(p.free[5]) == 1
