"""Host-side tests of the calls over several sequences (no GPU needed): every
argument error is reported with its documented status before anything is enqueued."""

import pytest
import torch

H = pytest.importorskip("paper_2605_06892_amd.hsa_step")

OK, NULL, SHAPE, BUDGET, DTYPE, ALIAS, WORKSPACE, LAUNCH = range(8)
F32, BF16, E4M3 = 0, 1, 2
# fake device addresses, far apart: never dereferenced, every call below fails validation first
P = [0x100000000000 + i * 0x10000000000 for i in range(12)]


@pytest.fixture(scope="module")
def lib():
    return H.lib()


def _call(f, base, **change):
    """The call with some of its named arguments changed."""
    args = dict(base, **change)
    return f(*args.values(), None)


STORE = dict(dtype=BF16, k=P[0], k_stride=1024, v=P[1], v_stride=1024, idx=P[2], n=10, n_rows=100, kv_heads=8,
             head_dim=128, cache_dtype=E4M3, k_cache=P[3], v_cache=P[4], k_exp=P[5], v_exp=P[6])

CACHE_REFUSALS = [
    (dict(dtype=2), DTYPE), (dict(dtype=9), DTYPE), (dict(cache_dtype=F32), DTYPE), (dict(cache_dtype=3), DTYPE),
    (dict(dtype=F32, cache_dtype=BF16), DTYPE),
    (dict(n=-1), SHAPE), (dict(n_rows=-1), SHAPE), (dict(n_rows=2 ** 31), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(kv_heads=-2 ** 31), SHAPE), (dict(kv_heads=2 ** 31 - 1), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(k_stride=1016), SHAPE), (dict(v_stride=1028), SHAPE),
    (dict(k_stride=2 ** 40), SHAPE), (dict(k_stride=-1024), SHAPE), (dict(n=2 ** 31 - 1), SHAPE),
    (dict(k=P[0] + 8), SHAPE), (dict(k_cache=P[3] + 8), SHAPE), (dict(idx=P[2] + 2), SHAPE),
    (dict(dtype=F32, k=P[0] + 2), SHAPE),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(idx=None), NULL), (dict(k_cache=None), NULL),
    (dict(v_cache=None), NULL), (dict(k_exp=None), NULL), (dict(v_exp=None), NULL),
    (dict(k=P[3]), ALIAS), (dict(v=P[4] + 1024), ALIAS), (dict(k=P[3] - 16), ALIAS),
]


@pytest.mark.parametrize("change,status", CACHE_REFUSALS + [
    (dict(v_cache=P[3]), ALIAS), (dict(k_exp=P[3] + 64), ALIAS), (dict(v_exp=P[5]), ALIAS), (dict(idx=P[4]), ALIAS)])
def test_store_refusals(lib, change, status):
    assert _call(lib.hsa_cache_store, STORE, **change) == status


def test_store_of_nothing(lib):
    assert _call(lib.hsa_cache_store, STORE, n=0, k=None, v=None, idx=None) == OK
    assert _call(lib.hsa_cache_store, STORE, n_rows=0, k_cache=None, v_cache=None, k_exp=None, v_exp=None) == OK


LOAD = dict(cache_dtype=E4M3, k_cache=P[3], v_cache=P[4], k_exp=P[5], v_exp=P[6], idx=P[2], n=10, n_rows=100, kv_heads=8,
            head_dim=128, dtype=BF16, k=P[0], k_stride=1024, v=P[1], v_stride=1024)


@pytest.mark.parametrize("change,status", CACHE_REFUSALS + [
    (dict(v=P[0]), ALIAS), (dict(idx=P[0] + 64), ALIAS), (dict(k=P[5]), ALIAS)])
def test_load_refusals(lib, change, status):
    assert _call(lib.hsa_cache_load, LOAD, **change) == status


def test_load_of_nothing(lib):
    assert _call(lib.hsa_cache_load, LOAD, n=0, k=None, v=None, idx=None) == OK


PACKED = dict(dtype=BF16, q=P[0], q_stride=2048, k=P[1], k_stride=512, v=P[2], v_stride=512, cu_q=P[3], cu_kv=P[4],
              n_seqs=3, n_q=100, n_kv=200, heads=16, kv_heads=4, head_dim=128, scale=0.1, causal=1, o=P[5], lse=P[6])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E4M3), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(kv_heads=3), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=-4), SHAPE),
    (dict(heads=-16, kv_heads=-4), SHAPE), (dict(head_dim=32), SHAPE), (dict(head_dim=256), SHAPE),
    (dict(n_seqs=-1), SHAPE), (dict(n_seqs=2 ** 31 - 1), SHAPE), (dict(n_q=-1), SHAPE), (dict(n_kv=-1), SHAPE),
    (dict(n_q=2 ** 31 - 1), SHAPE), (dict(n_q=2 ** 62), SHAPE), (dict(n_kv=2 ** 31), SHAPE), (dict(n_kv=2 ** 30 + 1), SHAPE),
    (dict(n_q=2 ** 24), SHAPE), (dict(n_seqs=2 ** 22), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(scale=float("nan")), SHAPE),
    (dict(q_stride=2040), SHAPE), (dict(k_stride=516), SHAPE), (dict(v_stride=0), SHAPE), (dict(q_stride=2 ** 23), SHAPE),
    (dict(q=P[0] + 4), SHAPE), (dict(o=P[5] + 8), SHAPE), (dict(lse=P[6] + 1), SHAPE), (dict(cu_q=P[3] + 2), SHAPE),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_q=None), NULL), (dict(cu_kv=None), NULL),
    (dict(o=None), NULL),
    (dict(o=P[0]), ALIAS), (dict(o=P[1] + 64), ALIAS), (dict(lse=P[5]), ALIAS), (dict(lse=P[2]), ALIAS),
    (dict(cu_kv=P[5] + 64), ALIAS),
])
def test_packed_refusals(lib, change, status):
    assert _call(lib.hsa_packed_attention, PACKED, **change) == status


def test_packed_of_nothing(lib):
    f = lib.hsa_packed_attention
    assert _call(f, PACKED, n_q=0, q=None, o=None) == OK
    assert _call(f, PACKED, n_seqs=0, cu_q=None, cu_kv=None) == OK


PAGED = dict(dtype=BF16, q=P[0], q_stride=2048, cache_dtype=E4M3, k_cache=P[1], v_cache=P[2], k_exp=P[3], v_exp=P[4],
             page_table=P[5], max_pages=100, kv_lens=P[6], n_seqs=3, n_pages=40, page_size=64, heads=16, kv_heads=4,
             head_dim=128, scale=0.1, o=P[7], lse=P[8], workspace=P[9], workspace_bytes=32 << 20)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=E4M3), DTYPE), (dict(cache_dtype=F32), DTYPE), (dict(cache_dtype=7), DTYPE),
    (dict(dtype=F32, cache_dtype=BF16), DTYPE),
    (dict(kv_heads=5), SHAPE), (dict(heads=0), SHAPE), (dict(head_dim=80), SHAPE), (dict(n_seqs=-1), SHAPE),
    (dict(n_seqs=2 ** 20), SHAPE), (dict(n_pages=-1), SHAPE), (dict(max_pages=-1), SHAPE), (dict(page_size=0), SHAPE),
    (dict(page_size=-64), SHAPE), (dict(n_pages=2 ** 30), SHAPE), (dict(max_pages=2 ** 24 + 1), SHAPE),
    (dict(page_size=2 ** 31 - 1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(q_stride=1024), SHAPE), (dict(q_stride=2052), SHAPE), (dict(q=P[0] + 2), SHAPE), (dict(k_cache=P[1] + 8), SHAPE),
    (dict(o=P[7] + 8), SHAPE), (dict(lse=P[8] + 2), SHAPE), (dict(page_table=P[5] + 1), SHAPE),
    (dict(kv_lens=P[6] + 2), SHAPE), (dict(workspace=P[9] + 8), SHAPE),
    (dict(q=None), NULL), (dict(k_cache=None), NULL), (dict(v_cache=None), NULL), (dict(k_exp=None), NULL),
    (dict(v_exp=None), NULL), (dict(page_table=None), NULL), (dict(kv_lens=None), NULL), (dict(o=None), NULL),
    (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE),
    (dict(o=P[0]), ALIAS), (dict(o=P[2] + 640), ALIAS), (dict(lse=P[7] + 64), ALIAS), (dict(workspace=P[1]), ALIAS),
    (dict(workspace=P[7] - 64), ALIAS), (dict(kv_lens=P[9]), ALIAS), (dict(page_table=P[8]), ALIAS),
])
def test_paged_refusals(lib, change, status):
    assert _call(lib.hsa_paged_attention, PAGED, **change) == status


def test_paged_of_nothing(lib):
    assert _call(lib.hsa_paged_attention, PAGED, n_seqs=0, q=None, o=None, workspace=None) == OK


def test_paged_workspace_bytes(lib):
    f = lib.hsa_paged_attention_workspace_bytes
    assert f(BF16, 1, 16, 2, 64, 768) == 0                  # too short to split
    for rows in (769, 1025, 2048, 2049, 7000):              # enough for fewer sequences and rows
        need = [f(BF16, n, 16, 2, 64, rows) for n in range(300)]
        assert need == sorted(need) and all(need[1:]) and f(BF16, 40, 16, 2, 64, rows - 1) <= need[40]
    assert 0 < f(BF16, 1, 16, 2, 64, 7000) < f(BF16, 64, 16, 2, 64, 7000)
    for args in [(BF16, 10000, 64, 8, 128, 2 ** 30), (F32, 1, 64, 64, 128, 2 ** 30), (BF16, 2, 1, 1, 64, 300)]:
        assert f(*args) <= 32 << 20 == H.PAGED_WORKSPACE_BYTES
    for args in [(E4M3, 1, 16, 2, 64, 700), (BF16, -1, 16, 2, 64, 700), (BF16, 1, 16, 3, 64, 700),
                 (BF16, 1, 16, 2, 65, 700), (BF16, 1, 16, 2, 64, -1), (BF16, 1, 16, 2, 64, 2 ** 31)]:
        assert f(*args) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        H.hsa_cache_store(x, x, i, 4, 2, x, x)
    with pytest.raises(ValueError):
        H.hsa_cache_load(x, x, i, 4, 2, x, x)
    with pytest.raises(ValueError):
        H.hsa_packed_attention(x, x, x, i, i, 2, 2, 128, 0.1, True, x)
    with pytest.raises(ValueError):
        H.hsa_paged_attention(x, x, x, i.view(4, 1), i, 16, 2, 2, 128, 0.1, x, None)


@pytest.mark.parametrize("scale,status", [(2.0 ** 127, OK), (2.0 ** 127 * (1 + 2.0 ** -23), SHAPE), (3.4028234e38, SHAPE)])
def test_scales_whose_product_with_log2_e_is_infinite(lib, scale, status):
    """The bf16 forms take scale * log2(e) in fp32: refused where that is not finite, and up to 2^127 it is."""
    # with nothing to do, so that the scale is all that is checked
    assert _call(lib.hsa_packed_attention, PACKED, n_seqs=0, scale=scale) == status
    assert _call(lib.hsa_paged_attention, PAGED, n_seqs=0, scale=scale) == status
