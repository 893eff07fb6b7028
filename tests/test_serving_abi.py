"""Host-side tests of the calls around a decoding step (no GPU needed): every argument error is
reported with its documented status before anything is enqueued."""

import pytest
import torch

H = pytest.importorskip("paper_2605_06892_amd.hsa_step")

OK, NULL, SHAPE, BUDGET, DTYPE, ALIAS, WORKSPACE, LAUNCH = range(8)
F32, BF16, E4M3, E2M1 = 0, 1, 2, 4
# fake device addresses, far apart: never dereferenced, every call below fails validation first
P = [0x100000000000 + i * 0x10000000000 for i in range(16)]


@pytest.fixture(scope="module")
def lib():
    return H.lib()


def _call(f, base, **change):
    return f(*dict(base, **change).values(), None)


STORE = dict(dtype=BF16, k=P[0], k_stride=1024, v=P[1], v_stride=1024, idx=P[2], n=10, n_rows=100, kv_heads=8,
             head_dim=128, cache_dtype=E2M1, k_cache=P[3], v_cache=P[4], k_exp=P[5], v_exp=P[6])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E2M1), DTYPE), (dict(cache_dtype=5), DTYPE), (dict(n=-1), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(k_cache=P[3] + 8), SHAPE), (dict(k_exp=None), NULL), (dict(v_exp=None), NULL),
    (dict(v_cache=P[3] + 51184), ALIAS),   # the caches' last 16 bytes: 100 rows of 512 bytes
    (dict(v_exp=P[5] + 3199), ALIAS),      # 100 rows of 32 exponents
    (dict(v_cache=P[5]), ALIAS)])
def test_store_refusals(lib, change, status):
    assert _call(lib.hsa_cache_store, STORE, **change) == status


def test_store_rows_side_by_side(lib):
    """Caches and exponents that end where the next begins do not overlap (nothing to do: n_rows of them, n = 0)."""
    assert _call(lib.hsa_cache_store, STORE, n=0) == OK


PAGED = dict(dtype=BF16, q=P[0], q_stride=2048, cache_dtype=E2M1, k_cache=P[1], v_cache=P[2], k_exp=P[3], v_exp=P[4],
             page_table=P[5], max_pages=100, kv_lens=P[6], n_seqs=3, n_pages=40, page_size=64, heads=16, kv_heads=4,
             head_dim=128, scale=0.1, o=P[7], lse=P[8], workspace=P[9], workspace_bytes=32 << 20)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E2M1), DTYPE), (dict(cache_dtype=3), DTYPE), (dict(k_exp=None), NULL), (dict(v_cache=P[2] + 4), SHAPE),
    (dict(o=P[1] + 40 * 64 * 256 - 16), ALIAS), (dict(lse=P[4] + 40 * 64 * 16 - 4), ALIAS)])
def test_paged_refusals(lib, change, status):
    assert _call(lib.hsa_paged_attention, PAGED, **change) == status


QUANTIZE = dict(dtype=BF16, w=P[0], w_stride=512, n_rows=100, d=512, codes=P[1], exps=P[2])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E2M1), DTYPE), (dict(dtype=-1), DTYPE), (dict(n_rows=-1), SHAPE), (dict(n_rows=2 ** 31), SHAPE),
    (dict(d=0), SHAPE), (dict(d=48), SHAPE), (dict(d=-32), SHAPE), (dict(d=2 ** 22 + 32, w_stride=2 ** 23), SHAPE),
    (dict(n_rows=2 ** 26), SHAPE), (dict(w_stride=504), SHAPE), (dict(w_stride=516), SHAPE), (dict(w_stride=-2 ** 63), SHAPE),
    (dict(w=P[0] + 2), SHAPE), (dict(codes=P[1] + 8), SHAPE), (dict(w=None), NULL), (dict(codes=None), NULL),
    (dict(exps=None), NULL), (dict(codes=P[0] + 1024), ALIAS), (dict(exps=P[1] + 25599), ALIAS), (dict(exps=P[0]), ALIAS)])
def test_quantize_refusals(lib, change, status):
    assert _call(lib.hsa_quantize_w4, QUANTIZE, **change) == status


def test_quantize_of_nothing(lib):
    assert _call(lib.hsa_quantize_w4, QUANTIZE, n_rows=0, w=None, codes=None, exps=None) == OK


LINEAR = dict(dtype=BF16, x=P[0], n_rows=4, d_in=512, w=P[1], w_exp=P[2], d_out=100, row_scale=P[3], residual=P[4], gelu=0,
              out_dtype=BF16, y=P[5])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E2M1), DTYPE), (dict(out_dtype=E4M3), DTYPE), (dict(dtype=F32), DTYPE), (dict(out_dtype=7), DTYPE),
    (dict(n_rows=-1), SHAPE), (dict(n_rows=2 ** 18 + 1), SHAPE), (dict(d_in=0), SHAPE), (dict(d_in=40), SHAPE),
    (dict(d_in=-32), SHAPE), (dict(d_in=2 ** 22 + 32), SHAPE), (dict(d_out=-1), SHAPE), (dict(d_out=2 ** 22 + 1), SHAPE),
    (dict(gelu=1), SHAPE), (dict(out_dtype=F32), SHAPE), (dict(out_dtype=F32, residual=None, gelu=1), SHAPE),
    (dict(x=P[0] + 8), SHAPE), (dict(w=P[1] + 8), SHAPE), (dict(y=P[5] + 4), SHAPE), (dict(residual=P[4] + 8), SHAPE),
    (dict(row_scale=P[3] + 2), SHAPE),
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(w_exp=None), NULL), (dict(y=None), NULL),
    (dict(y=P[0] + 64), ALIAS), (dict(y=P[1] + 25584), ALIAS), (dict(y=P[2] + 1584), ALIAS), (dict(row_scale=P[5] + 796), ALIAS),
    (dict(residual=P[5] + 16), ALIAS)])
def test_linear_refusals(lib, change, status):
    assert _call(lib.hsa_linear_w4, LINEAR, **change) == status


def test_linear_of_nothing(lib):
    assert _call(lib.hsa_linear_w4, LINEAR, n_rows=0, x=None, y=None) == OK
    assert _call(lib.hsa_linear_w4, LINEAR, d_out=0, w=None, w_exp=None, y=None) == OK


NORM = dict(dtype=BF16, q=P[0], q_stride=2560, k=P[1], k_stride=2560, n=10, heads=16, kv_heads=4, head_dim=128, q_weight=P[2],
            k_weight=P[3], eps=1e-6, rope=P[4], n_pos=100, rope_dim=128, interleaved=0, pos=P[5], q_out=P[6], q_out_stride=2048,
            k_out=P[7], k_out_stride=512)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E4M3), DTYPE), (dict(n=-1), SHAPE), (dict(n=2 ** 31 - 1), SHAPE), (dict(heads=-1), SHAPE), (dict(kv_heads=-1), SHAPE),
    (dict(heads=2 ** 16), SHAPE), (dict(heads=2 ** 31 - 1, kv_heads=2 ** 31 - 1), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(eps=0.0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(n_pos=-1), SHAPE), (dict(n_pos=2 ** 31), SHAPE), (dict(rope_dim=-8), SHAPE), (dict(rope_dim=136), SHAPE),
    (dict(rope_dim=12), SHAPE), (dict(q_stride=2040), SHAPE), (dict(k_stride=516), SHAPE), (dict(q_out_stride=2 ** 23), SHAPE),
    (dict(k_out_stride=-512), SHAPE), (dict(q=P[0] + 8), SHAPE), (dict(k_out=P[7] + 4), SHAPE), (dict(q_weight=P[2] + 2), SHAPE),
    (dict(rope=P[4] + 8), SHAPE), (dict(pos=P[5] + 1), SHAPE),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(q_out=None), NULL), (dict(k_out=None), NULL), (dict(rope=None), NULL),
    (dict(q_out=P[0]), ALIAS), (dict(q_out=P[0], q_out_stride=2560, k=P[0] + 2048), ALIAS),  # keys inside the query rows
    (dict(q_out=P[1] + 1040, q_out_stride=2560), ALIAS),      # reaches into the next row's keys
    (dict(k_out=P[6] + 64), ALIAS), (dict(k_out=P[4]), ALIAS), (dict(q_out=P[5] - 64), ALIAS), (dict(k_out=P[2] + 240), ALIAS),
    (dict(q=P[7]), ALIAS)])
def test_norm_refusals(lib, change, status):
    assert _call(lib.hsa_qk_norm_rope, NORM, **change) == status


def test_norm_of_nothing(lib):
    f = lib.hsa_qk_norm_rope
    assert _call(f, NORM, n=0, q=None, k=None, q_out=None, k_out=None, rope=None) == OK
    assert _call(f, NORM, heads=0, kv_heads=0) == OK


PLAN = dict(past=P[0], fresh=P[1], n_seqs=10, page_size=16, max_pages=8, page_table=P[2], free_pages=P[3], n_free=100, free_at=P[4],
            n_tokens=50, cu=P[5], kv_lens=P[6], pos=P[7], slots=P[8], free_next=P[9])


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=-1), SHAPE), (dict(n_seqs=2 ** 31 - 1), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=-16), SHAPE),
    (dict(max_pages=-1), SHAPE), (dict(max_pages=2 ** 27), SHAPE), (dict(page_size=2 ** 31 - 1), SHAPE), (dict(n_free=-1), SHAPE),
    (dict(n_free=2 ** 30 + 1), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=2 ** 30), SHAPE),
    (dict(past=P[0] + 2), SHAPE), (dict(slots=P[8] + 1), SHAPE),
    (dict(past=None), NULL), (dict(fresh=None), NULL), (dict(page_table=None), NULL), (dict(free_pages=None), NULL),
    (dict(free_at=None), NULL), (dict(cu=None), NULL), (dict(kv_lens=None), NULL), (dict(pos=None), NULL), (dict(slots=None), NULL),
    (dict(free_next=None), NULL),
    (dict(pos=P[8] + 196), ALIAS), (dict(cu=P[0]), ALIAS), (dict(kv_lens=P[0] + 4), ALIAS), (dict(kv_lens=P[1]), ALIAS),
    (dict(free_next=P[4] + 4), ALIAS), (dict(page_table=P[3] + 396), ALIAS), (dict(slots=P[2] + 316), ALIAS),
    (dict(free_next=P[5] + 40), ALIAS)])
def test_plan_refusals(lib, change, status):
    assert _call(lib.hsa_page_plan, PLAN, **change) == status


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    c, e, i = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        H.hsa_quantize_w4(x, c, e)
    with pytest.raises(ValueError):
        H.hsa_linear_w4(x, 4, c, e, x)
    with pytest.raises(ValueError):
        H.hsa_qk_norm_rope(x, x, 2, 2, 128, x, x)
    with pytest.raises(ValueError):
        H.hsa_page_plan(i, i, 16, i.view(4, 1), i, i, i, i, i, i, i)
    with pytest.raises(ValueError):
        H.hsa_cache_store(x, x, i, 4, 2, c, c, e, e)
