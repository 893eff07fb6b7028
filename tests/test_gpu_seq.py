"""GPU tests of the calls over several sequences, against definitions in 64 bits.

Tolerances, per output element, from the arithmetic (u = 2^-24, a half step of fp32):
  - a score is a sum of head_dim products in fp32: off by at most (head_dim + 4) u S, with
    S = scale * max_j sum_c |q_c k_jc|, and its probability by that share of itself, twice (its own
    and in the normalizing sum);
  - sums over n keys add n u, exponentials, rescalings and the division some 64 u of
    A = sum_j p_j |v_j|;
  - the bf16 form rounds probabilities (2^-8 of each, so 2^-8 A) and the output (2^-8 of it);
  - lse is off by the score's error, the sum's, and a few roundings of itself.
"""

import math

import numpy as np
import pytest
import torch

from gpu_util import Guarded
from paper_2605_06892_amd import hsa_step as H
from paper_2605_06892_amd import paged

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
T = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g)


def attend64(q, k, v, seen, scale):
    """One head in 64 bits: q [m, dh], k and v [n, dh], seen bool [m, n]. Rows that see nothing: 0 and -inf.
    Returns o, lse, A (sum p |v|) and S (the greatest sum of magnitudes behind a score)."""
    q, k, v = q.double(), k.double(), v.double()
    m, dh = q.shape
    if k.shape[0] == 0:
        return torch.zeros(m, dh).double(), torch.full((m,), -math.inf).double(), torch.zeros(m, dh).double(), 0.0
    s = (q @ k.t()) * scale
    s = torch.where(seen, s, torch.tensor(-math.inf).double())
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    p = torch.where(seen, p, torch.zeros_like(p))
    return p @ v, lse, p @ v.abs(), float((q.abs() @ k.abs().t()).max() * scale)


def check(got, lse_got, want, lse_want, A, S, dtype, n_keys, dh):
    score = 2 * (dh + 4) * U * S
    bar = (2 * score + (n_keys + 64) * U) * A + 2 * U * want.abs() + 1e-30
    if dtype == "bf16":
        bar = bar + 2.0 ** -8 * (A + want.abs()) * (1 + 2.0 ** -7)
    off = (got.cpu().double() - want).abs()
    worst = float((off / bar).max()) if off.numel() else 0.0
    assert worst <= 1, f"{worst:.2f} of the bound"
    if lse_got is not None:
        none = torch.isinf(lse_want)
        lg = lse_got.cpu().double()
        assert torch.equal(none, torch.isinf(lg)) and torch.all(lg[none] < 0)
        d = (lg - lse_want)[~none].abs()
        lbar = score + (n_keys + 64) * U + 8 * U * lse_want[~none].abs()
        assert torch.all(d <= lbar), float((d / lbar).max())


# ---------------------------------------------------------------- packed


@pytest.fixture(params=[("bf16", ""), ("bf16", "16x8"), ("bf16", "16x4"), ("bf16", "32x8"), ("bf16", "32x4"),
                        ("bf16", "128x4"), ("bf16", "256x8"), ("f32", "16x8"), ("f32", "16x4")],
                ids=lambda p: "-".join(filter(None, p)))
def form(request, monkeypatch):
    """The dtype, with every tile (rows x waves) whatever the launch would choose."""
    dtype, tile = request.param
    if tile:
        monkeypatch.setenv("HSA_PACKED_TILE", tile)
    return dtype


def packed_inputs(seed, dtype, lens_q, lens_k, heads, kv, dh, lead=0, tail=0, fused=False):
    """q, k, v on the host with `lead` rows before the first sequence and `tail` after the last, and the offsets."""
    g = _gen(seed)
    n_q, n_k = lead + sum(lens_q) + tail, lead + sum(lens_k) + tail
    q, k, v = (_randn(g, n, w * dh).to(T[dtype]) for n, w in ((n_q, heads), (n_k, kv), (n_k, kv)))
    cu_q = torch.tensor(np.cumsum([lead] + list(lens_q)), dtype=torch.int32)
    cu_k = torch.tensor(np.cumsum([lead] + list(lens_k)), dtype=torch.int32)
    return q, k, v, cu_q, cu_k


def packed_want(q, k, v, cu_q, cu_k, heads, kv, dh, scale, causal):
    """o, lse, A over the rows of the sequences, NaN elsewhere, and S."""
    n_q = q.shape[0]
    o, A = (torch.full((n_q, heads * dh), math.nan).double() for _ in range(2))
    lse = torch.full((n_q, heads), math.nan).double()
    S = 0.0
    for s in range(len(cu_q) - 1):
        a, b, c, d = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        m, n = b - a, d - c
        seen = torch.ones(m, n, dtype=torch.bool)
        if causal:
            seen = torch.arange(n)[None] <= torch.arange(m)[:, None] + (n - m)
        for h in range(heads):
            hk = h // (heads // kv)
            x, l, y, sm = attend64(q[a:b, h * dh:(h + 1) * dh], k[c:d, hk * dh:(hk + 1) * dh],
                                   v[c:d, hk * dh:(hk + 1) * dh], seen, scale)
            o[a:b, h * dh:(h + 1) * dh], A[a:b, h * dh:(h + 1) * dh], lse[a:b, h] = x, y, l
            S = max(S, sm)
    return o, lse, A, S


def run_packed(q, k, v, cu_q, cu_k, heads, kv, dh, scale, causal, o=None, lse=None, **kw):
    o = torch.empty_like(q, device=DEV, memory_format=torch.contiguous_format) if o is None else o
    lse = torch.empty(q.shape[0], heads, device=DEV) if lse is None else lse
    H.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), cu_q.to(DEV), cu_k.to(DEV), heads, kv, dh, scale, causal, o,
                           lse=lse, **kw)
    return o, lse


PACKED = [
    # lens_q, lens_kv, heads, kv_heads
    ([1], [1], 1, 1),
    ([1], [300], 4, 4),
    ([17], [17], 2, 1),
    ([5, 0, 64, 1, 33], [5, 0, 64, 1, 33], 6, 2),
    ([31, 100], [95, 100], 3, 3),                  # rows before the queries (a prompt continued)
    ([40, 7, 3], [9, 0, 3], 4, 2),                 # more queries than keys: rows that see none
    ([129, 257, 2], [129, 257, 2], 8, 1),
    ([70, 3], [70, 3], 7, 1),
    ([260], [700], 5, 5),
    ([12, 13], [500, 31], 32, 2),
    ([1100], [1100], 8, 4),
    ([300, 513], [300, 800], 16, 8),
]


@pytest.mark.parametrize("lens_q,lens_k,heads,kv", PACKED, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
def test_packed(form, dh, causal, lens_q, lens_k, heads, kv):
    dtype = form
    q, k, v, cu_q, cu_k = packed_inputs(len(lens_q) * 100 + sum(lens_q), dtype, lens_q, lens_k, heads, kv, dh, 3, 5)
    scale = dh ** -0.5
    o, lse = Guarded(q.shape, T[dtype], 1), Guarded((q.shape[0], heads), torch.float32, 2)
    o.t.fill_(7.0)
    lse.t.fill_(7.0)
    run_packed(q, k, v, cu_q, cu_k, heads, kv, dh, scale, causal, o.t, lse.t)
    want, lse_want, A, S = packed_want(q, k, v, cu_q, cu_k, heads, kv, dh, scale, causal)
    rows = slice(3, 3 + sum(lens_q))
    check(o.t[rows], lse.t[rows], want[rows], lse_want[rows], A[rows], S, dtype, max(lens_k), dh)
    o.check("o")
    lse.check("lse")
    for x in (o.t, lse.t):  # rows of no sequence are left as they were
        assert torch.all(x[:3] == 7.0) and torch.all(x[rows.stop:] == 7.0)


def test_packed_many_sequences(form):
    dtype = form
    lens = [(i * 7) % 23 for i in range(150)]
    q, k, v, cu_q, cu_k = packed_inputs(3, dtype, lens, lens, 4, 2, 64)
    o, lse = run_packed(q, k, v, cu_q, cu_k, 4, 2, 64, 0.125, True)
    want, lw, A, S = packed_want(q, k, v, cu_q, cu_k, 4, 2, 64, 0.125, True)
    check(o, lse, want, lw, A, S, dtype, 23, 64)


@pytest.mark.parametrize("causal", [True, False])
def test_packed_thousands_of_sequences(form, causal):
    """More than 64 x 64 of them, of no to 3 tokens, behind rows of no sequence."""
    dtype = form
    lens = [(i * 7) % 4 for i in range(4500)]
    q, k, v, cu_q, cu_k = packed_inputs(4, dtype, lens, lens, 2, 1, 64, 37, 5)
    o, lse = (torch.full((q.shape[0], w), 7.0, dtype=t, device=DEV) for w, t in ((128, T[dtype]), (2, torch.float32)))
    run_packed(q, k, v, cu_q, cu_k, 2, 1, 64, 0.125, causal, o, lse)
    want, lw, A, S = packed_want(q, k, v, cu_q, cu_k, 2, 1, 64, 0.125, causal)
    rows = slice(37, 37 + sum(lens))
    check(o[rows], lse[rows], want[rows], lw[rows], A[rows], S, dtype, 3, 64)
    assert torch.all(o[:37] == 7.0) and torch.all(o[rows.stop:] == 7.0)


def test_packed_without_keys(form):
    dtype = form
    q = torch.ones(5, 128, dtype=T[dtype], device=DEV)
    k = torch.empty(0, 128, dtype=T[dtype], device=DEV)
    cu = torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV)
    o, lse = torch.full_like(q, 7.0), torch.full((5, 1), 7.0, device=DEV)
    H.hsa_packed_attention(q, k, k, cu, torch.zeros_like(cu), 1, 1, 128, 0.1, False, o, lse=lse)
    assert torch.all(o == 0) and torch.all(lse == -math.inf)
    H.hsa_packed_attention(q[:0], k, k, cu, cu, 1, 1, 128, 0.1, False, o[:0])           # no queries
    H.hsa_packed_attention(q, k, k, cu[:1], cu[:1], 1, 1, 128, 0.1, False, o.fill_(7.0))  # no sequences
    assert torch.all(o == 7.0)


def off_by_one(t):
    """The tensor at an address that is a multiple of 4 bytes and no more."""
    raw = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
    x = raw[1:].view(t.shape)
    x.copy_(t)
    return x


def test_f32_rows_of_4_byte_alignment():
    """fp32 tensors off the 16-byte alignment, through every call."""
    heads, kv, dh, n, page = 4, 2, 64, 150, 8
    g = _gen(21)
    q, k, v = (off_by_one(_randn(g, n, w * dh)) for w in (heads, kv, kv))
    cu = torch.tensor([0, 47, n], dtype=torch.int32)
    o, lse = off_by_one(torch.zeros(n, heads * dh)), torch.empty(n, heads, device=DEV)
    cud = cu.to(DEV)
    H.hsa_packed_attention(q, k, v, cud, cud, heads, kv, dh, 0.125, True, o, lse=lse)
    want, lw, A, S = packed_want(q.cpu(), k.cpu(), v.cpu(), cu, cu, heads, kv, dh, 0.125, True)
    check(o, lse, want, lw, A, S, "f32", n, dh)
    kc, vc = (off_by_one(torch.zeros(160, kv * dh)) for _ in range(2))
    idx = torch.randperm(160, generator=g)[:n].to(torch.int32)
    H.hsa_cache_store(k, v, idx.to(DEV), n, kv, kc, vc)
    k2, v2 = (off_by_one(torch.zeros(n, kv * dh)) for _ in range(2))
    H.hsa_cache_load(kc, vc, idx.to(DEV), n, kv, k2, v2)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    table = torch.randperm(20, generator=g).view(1, 20).to(torch.int32)
    o1, l1 = run_paged(off_by_one(q[:1].cpu()), (kc, vc, None, None), table, [155], page, heads, kv, dh, 0.125)
    want, lw, A, S = paged_want(q[:1].cpu(), kc.cpu(), vc.cpu(), table, [155], page, 20, heads, kv, dh, 0.125)
    check(o1, l1, want, lw, A, S, "f32", 155, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_packed_strided_rows_and_other_stream(dtype, dh):
    """Slices of one projection's output, on a stream of their own."""
    lens, heads, kv = [45, 200, 1], 6, 3
    g = _gen(11)
    qkv = _randn(g, sum(lens), (heads + 2 * kv) * dh).to(T[dtype])
    q, k, v = qkv.split([heads * dh, kv * dh, kv * dh], dim=1)
    cu = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32)
    dev = qkv.to(DEV)
    qd, kd, vd = dev.split([heads * dh, kv * dh, kv * dh], dim=1)
    o = torch.empty(sum(lens), heads * dh, dtype=T[dtype], device=DEV)
    cud = cu.to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    H.hsa_packed_attention(qd, kd, vd, cud, cud, heads, kv, dh, dh ** -0.5, True, o, stream=s)
    s.synchronize()
    want, lw, A, S = packed_want(q, k, v, cu, cu, heads, kv, dh, dh ** -0.5, True)
    check(o, None, want, lw, A, S, dtype, 200, dh)


@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lens", [[40, 300, 20], [600, 9]])
def test_packed_odd_values_stay_in_what_sees_them(form, dh, odd, lens):
    """Keys and values that are not finite reach the rows that see them and no other: the rows before them under a
    causal mask, and the neighbouring sequences, are as without them, bit for bit."""
    dtype = form
    heads, kv, scale = 6, 2, dh ** -0.5
    q, k, v, cu, _ = packed_inputs(5, dtype, lens, lens, heads, kv, dh)
    o0, l0 = run_packed(q, k, v, cu, cu, heads, kv, dh, scale, True)
    at = int(cu[1]) - 7  # row of the first sequence
    v2, k2 = v.clone(), k.clone()
    v2[at, 3] = odd
    v2[at + 2, dh + 5] = odd
    k2[at + 4] = math.nan
    o1, l1 = run_packed(q, k2, v2, cu, cu, heads, kv, dh, scale, True)
    o0, o1, l0, l1 = o0.cpu(), o1.cpu(), l0.cpu(), l1.cpu()
    g = heads // kv * dh
    clean = torch.ones(o0.shape, dtype=torch.bool)
    clean[at:cu[1], 3:g:dh] = False            # the channel of the first odd value, in its group's heads
    clean[at + 2:cu[1], g + 5::dh] = False
    clean[at + 4:cu[1]] = False                # a NaN key: every channel of the rows that see it
    assert torch.equal(o0[clean], o1[clean])
    seen = o1[at:at + 2, 3:g:dh]
    assert torch.all(torch.isnan(seen) if math.isnan(odd) else seen == odd)
    seen = o1[at + 2:at + 4, g + 5::dh]
    assert torch.all(torch.isnan(seen) if math.isnan(odd) else seen == odd)
    assert torch.isnan(o1[at + 4:cu[1]]).all() and torch.isnan(l1[at + 4:cu[1]]).all()
    assert torch.equal(l0[:at + 4], l1[:at + 4]) and torch.equal(l0[cu[1]:], l1[cu[1]:])


def test_packed_infinite_last_value(form):
    """The last key of a sequence whose length is no multiple of anything, with an infinite value, without a mask."""
    dtype = form
    q, k, v, cu, _ = packed_inputs(6, dtype, [333], [333], 2, 2, 64)
    v[332, 7] = math.inf
    o, _ = run_packed(q, k, v, cu, cu, 2, 2, 64, 0.125, False)
    assert torch.all(o[:, 7] == math.inf) and torch.isfinite(o[:, :7]).all() and torch.isfinite(o[:, 8:]).all()


def test_packed_large_and_infinite_scores(form):
    """Scores thousands apart and of either sign, and scores of -infinity."""
    dtype = form
    lens = [50, 400]
    q, k, v, cu, _ = packed_inputs(7, dtype, lens, lens, 4, 2, 64)
    q = q * 300
    k[60:200, 0] = math.inf
    q[:, ::64] = -1.0  # channel 0 of every head: those keys' scores are -inf in every head of the first kv head
    o, lse = run_packed(q, k, v, cu, cu, 4, 2, 64, 0.125, True)
    keep = torch.ones(450, dtype=torch.bool)
    keep[60:200] = False
    for s, (a, b) in enumerate(((0, 50), (50, 450))):
        n = b - a
        seen = torch.arange(n)[None] <= torch.arange(n)[:, None]
        for h in range(4):
            hk = h // 2
            kk, sk = k[a:b, hk * 64:hk * 64 + 64], seen
            if hk == 0:
                sk = seen & keep[a:b][None]
                kk = torch.where(torch.isinf(kk), torch.zeros_like(kk), kk)
            c = slice(h * 64, h * 64 + 64)
            want, lw, A, S = attend64(q[a:b, c], kk, v[a:b, hk * 64:hk * 64 + 64], sk, 0.125)
            check(o[a:b, c], lse[a:b, h:h + 1], want, lw[:, None], A, S, dtype, n, 64)


def test_packed_offsets_out_of_range_or_order(form):
    """Offsets past the rows are clamped to them; nothing outside the buffers is touched whatever they hold."""
    dtype = form
    q, k, v, _, _ = packed_inputs(8, dtype, [100], [120], 4, 2, 64)
    o = Guarded(q.shape, T[dtype], 3)
    o.t.fill_(7.0)
    cu_q = torch.tensor([0, 40, 2 ** 31 - 1], dtype=torch.int32)
    cu_k = torch.tensor([-5, 50, 2 ** 30], dtype=torch.int32)
    run_packed(q, k, v, cu_q, cu_k, 4, 2, 64, 0.125, False, o.t)
    want, lw, A, S = packed_want(q, k, v, [0, 40, 100], [0, 50, 120], 4, 2, 64, 0.125, False)
    check(o.t, None, want, lw, A, S, dtype, 120, 64)
    for cu_q, cu_k in (([90, 10, 100, -3, 70], [0, 100, 20, 30, 5]), ([0, 100, 0, 100, 0], [120, 0, 120, 0, 120])):
        run_packed(q, k, v, torch.tensor(cu_q, dtype=torch.int32), torch.tensor(cu_k, dtype=torch.int32), 4, 2, 64, 0.125,
                   True, o.t)
        o.check("o")


def test_packed_refusals_of_the_binding():
    q = torch.zeros(8, 256, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(8, 128, dtype=torch.bfloat16, device=DEV)
    cu = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    o = torch.empty_like(q)
    ok = dict(q=q, k=k, v=k, cu_q=cu, cu_kv=cu, heads=2, kv_heads=1, head_dim=128, scale=0.1, causal=True, o=o)
    H.hsa_packed_attention(**ok)
    for change in (dict(q=q.t()), dict(cu_kv=cu[:1]), dict(o=o[:4]), dict(heads=4), dict(k=k[:, :64]), dict(o=o.view(-1))):
        with pytest.raises(ValueError):
            H.hsa_packed_attention(**{**ok, **change})
    for change in (dict(cu_q=cu.long()), dict(o=o.float()), dict(lse=torch.empty(8, 1, device=DEV)), dict(q=q.half())):
        with pytest.raises(TypeError):
            H.hsa_packed_attention(**{**ok, **change})
    with pytest.raises(H.HsaStepError):
        H.hsa_packed_attention(**{**ok, "o": q})


# ---------------------------------------------------------------- cache rows


def quantize64(x, kv):
    """Codes' values and exponents by the definition, in 64 bits: x [n, kv * dh] on the host."""
    y = x.double().view(x.shape[0], kv, -1).numpy()
    fin = np.where(np.isfinite(y), np.abs(y), 0.0)
    top = fin.max(-1)
    e = np.full(top.shape, -117, dtype=np.int64)
    for x_ in range(-117, 120):
        e = np.where(top > 448.0 * 2.0 ** (e.astype(np.float64)), np.minimum(e + 1, 119), e)
    z = y * 2.0 ** (-e[..., None].astype(np.float64))
    with np.errstate(invalid="ignore", divide="ignore"):
        mag = np.where(np.isfinite(z), np.abs(z), 0.0)
        binade = np.floor(np.log2(np.maximum(mag, 2.0 ** -6)))
        step = 2.0 ** (binade - 3)
        r = np.minimum(np.rint(mag / step) * step, 448.0)  # rint: ties to even
    r = np.where(np.isfinite(y), np.copysign(r, z), np.nan)
    return torch.from_numpy(r.reshape(x.shape)), torch.from_numpy(e)


def odd_rows(g, dtype, n, d, dh):
    """Rows of every kind: ordinary, tiny, huge, zero, on the ties of e4m3, at the limits, not finite."""
    x = _randn(g, n, d)
    x *= torch.exp(_randn(g, n, 1) * 20).clamp(1e-38, 1e37)
    x[::7, ::5] *= 100
    kinds = [torch.zeros(d), torch.full((d,), 448.0), torch.full((d,), 449.0),
             torch.arange(d) / 16.0, (torch.arange(d) % 64 + 0.5) * 2.0 ** -9, torch.full((d,), 1e-40),
             torch.full((d,), 3.3e38), -torch.full((d,), 3.38e38), torch.full((d,), 2.0 ** -126),
             torch.arange(d) * 2.0 ** -130, torch.where(torch.arange(d) % 3 == 0, math.inf, 1.5),
             torch.where(torch.arange(d) % 5 == 0, math.nan, -2.5), torch.full((d,), -math.inf), torch.full((d,), math.nan),
             torch.where(torch.arange(d) % dh == 1, 1.75 * 2.0 ** 127, 1.0), torch.full((d,), -0.0)]
    for i, row in enumerate(kinds):
        if i < n:
            x[i] = row
    return x.to(T[dtype])


def same(a, b):
    """Equal values, NaN equal to NaN."""
    a, b = a.cpu().double(), b.cpu().double()
    return bool(torch.all((a == b) | (torch.isnan(a) & torch.isnan(b))))


def exps(kv, n):
    return torch.full((n, kv), 33, dtype=torch.int8, device=DEV)


@pytest.mark.parametrize("n,n_rows,kv", [(1, 1, 1), (3, 9, 5), (40, 64, 3), (16, 4096, 8), (777, 1000, 12), (2049, 2049, 2)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_and_load_e4m3(dtype, dh, n, n_rows, kv):
    g = _gen(n * 10 + kv)
    d = kv * dh
    kvs = torch.cat([odd_rows(g, dtype, n, d, dh), _randn(g, n, d).to(T[dtype])], 1)  # keys beside values
    k, v = kvs[:, :d], kvs[:, d:]
    idx = torch.randperm(n_rows, generator=g)[:n].to(torch.int32)
    if n > 2:
        idx[2] = -1
    caches = [Guarded((n_rows, d), torch.uint8, s) for s in (1, 2)]
    es = [Guarded((n_rows, kv), torch.int8, s) for s in (3, 4)]
    for c in caches:
        c.t.fill_(0x55)
    for e in es:
        e.t.fill_(33)
    kd = kvs.to(DEV)
    kc, vc = (c.t.view(F8) for c in caches)
    idx_d = idx.to(DEV)
    H.hsa_cache_store(kd[:, :d], kd[:, d:], idx_d, n, kv, kc, vc, es[0].t, es[1].t)
    live = idx >= 0
    rows = idx[live].long()
    rest = torch.ones(n_rows, dtype=torch.bool)
    rest[rows] = False
    back = [torch.full((n + 1, d), 7.0, dtype=T[dtype], device=DEV) for _ in range(2)]
    H.hsa_cache_load(kc, vc, idx_d, n, kv, back[0], back[1], es[0].t, es[1].t)
    for x, c, e, b, name in zip((k, v), caches, es, back, "kv"):
        codes, ex = quantize64(x, kv)
        assert torch.equal(e.t.cpu()[rows].long(), ex[live]), name
        assert same(c.t.view(F8)[rows.to(DEV)].float() if n_rows else codes, codes[live]), name
        assert torch.all(c.t.cpu()[rest] == 0x55) and torch.all(e.t.cpu()[rest] == 33)
        c.check(name)
        e.check(name + "_exp")
        value = (codes.view(n, kv, dh) * torch.pow(2.0, ex.double())[..., None]).view(n, d)
        value[~live] = 0.0  # an index outside the cache reads zeros
        assert same(b[:n], value), name
        assert torch.all(b[n] == 7.0)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_and_load_unquantized(dtype, dh):
    g = _gen(9)
    n, n_rows, kv = 333, 500, 3
    d = kv * dh
    k, v = _randn(g, n, d).to(T[dtype]), _randn(g, n, d).to(T[dtype])
    k[3, 5], v[4, 6] = math.nan, math.inf
    idx = torch.randperm(n_rows, generator=g)[:n].to(torch.int32)
    idx[7], idx[8] = n_rows, -2 ** 31
    kc, vc = (torch.full((n_rows, d), 7.0, dtype=T[dtype], device=DEV) for _ in range(2))
    H.hsa_cache_store(k.to(DEV), v.to(DEV), idx.to(DEV), n, kv, kc, vc)
    live = (idx >= 0) & (idx < n_rows)
    want_k, want_v = (torch.full((n_rows, d), 7.0, dtype=T[dtype]) for _ in range(2))
    want_k[idx[live].long()], want_v[idx[live].long()] = k[live], v[live]
    assert same(kc, want_k) and same(vc, want_v)
    twice = torch.cat([idx, idx]).to(DEV)  # the same rows twice
    # into slices of a wider buffer
    wide = torch.full((2 * n, 2 * d + 64), 7.0, dtype=T[dtype], device=DEV)
    H.hsa_cache_load(kc, vc, twice, 2 * n, kv, wide[:, :d], torch.empty(2 * n, d, dtype=T[dtype], device=DEV))
    k[~live] = 0.0
    assert same(wide[:n, :d], k) and same(wide[n:, :d], k) and torch.all(wide[:, d:] == 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_reads_back(dtype):
    """All 256 codes at every exponent that the store may write."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(237, 1)
    ex = torch.arange(-117, 120, dtype=torch.int8)[:, None].repeat(1, 4)
    kc = codes.view(F8).to(DEV)
    idx = torch.arange(237, dtype=torch.int32, device=DEV)
    k, v = (torch.empty(237, 256, dtype=T[dtype], device=DEV) for _ in range(2))
    H.hsa_cache_load(kc, kc.clone(), idx, 237, 4, k, v, ex.to(DEV), ex.to(DEV))
    b = codes.long()
    e, f = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.pow(2.0, (e - 10).double()))
    mag = torch.where((b & 127) == 127, math.nan, mag)
    value = torch.where(b >= 128, -mag, mag) * torch.pow(2.0, ex.double()).repeat_interleave(64, 1)
    assert same(k, value) and same(v, value)


def test_cache_refusals_of_the_binding():
    k = torch.zeros(8, 256, dtype=torch.bfloat16, device=DEV)
    c = torch.zeros(16, 256, dtype=torch.uint8, device=DEV).view(F8)
    e = torch.zeros(16, 2, dtype=torch.int8, device=DEV)
    i = torch.arange(8, dtype=torch.int32, device=DEV)
    ok = dict(k=k, v=k, idx=i, n=8, kv_heads=2, k_cache=c, v_cache=c.clone(), k_exp=e, v_exp=e.clone())
    H.hsa_cache_store(**ok)
    for change in (dict(n=9), dict(k=k[:, :128]), dict(k=k.t()), dict(kv_heads=2, k=k[:4])):
        with pytest.raises(ValueError):
            H.hsa_cache_store(**{**ok, **change})
    for change in (dict(k_exp=None), dict(k_exp=e[:4]), dict(idx=i.long()), dict(v_cache=c[:3]), dict(k=k.float()),
                   dict(kv_heads=3), dict(k_cache=k, v_cache=k.float()), dict(k_cache=k.float(), v_cache=k.float())):
        with pytest.raises(TypeError):
            H.hsa_cache_store(**{**ok, **change})
    for change in (dict(v_cache=c), dict(k_exp=e, v_exp=e)):
        with pytest.raises(H.HsaStepError):
            H.hsa_cache_store(**{**ok, **change})
    ok.update(k=k, v=k.clone())
    H.hsa_cache_load(**ok)
    with pytest.raises(H.HsaStepError):
        H.hsa_cache_load(**{**ok, "v": k})


# ---------------------------------------------------------------- paged


def paged_inputs(seed, dtype, cache, lens, page, heads, kv, dh, spare=2, max_pages=None):
    """A cache of shuffled pages on the host: values, what the cache holds, the exponents, the table."""
    g = _gen(seed)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    width = max(need + [1]) + 1 if max_pages is None else max_pages
    perm = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = perm[at:at + m]
        at += m
    k, v = (_randn(g, n_pages * page, kv * dh).to(T[dtype]) for _ in range(2))
    q = _randn(g, len(lens), heads * dh).to(T[dtype])
    if cache != "e4m3":
        return q, k, v, (k, v, None, None), table
    held, value = [], []
    for x in (k, v):
        codes, ex = quantize64(x, kv)
        held.append((codes.float().to(F8), ex.to(torch.int8)))
        value.append((codes.view(-1, kv, dh) * torch.pow(2.0, ex.double())[..., None]).view(x.shape))
    return q, value[0], value[1], (held[0][0], held[1][0], held[0][1], held[1][1]), table


def paged_want(q, k, v, table, lens, page, n_pages, heads, kv, dh, scale):
    n = len(lens)
    o, A = (torch.zeros(n, heads * dh).double() for _ in range(2))
    lse = torch.empty(n, heads).double()
    S = 0.0
    for s in range(n):
        t = torch.arange(lens[s])
        pages = table[s].long()[t // page]
        ok = (pages >= 0) & (pages < n_pages)
        rows = (pages * page + t % page)[ok]
        for h in range(heads):
            c, ck = slice(h * dh, (h + 1) * dh), slice(h // (heads // kv) * dh, (h // (heads // kv) + 1) * dh)
            x, l, y, sm = attend64(q[s:s + 1, c], k[rows][:, ck], v[rows][:, ck], torch.ones(1, len(rows), dtype=torch.bool),
                                   scale)
            o[s, c], A[s, c], lse[s, h] = x[0], y[0], l[0]
            S = max(S, sm)
    return o, lse, A, S


def run_paged(q, held, table, lens, page, heads, kv, dh, scale, o=None, ws=None, **kw):
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    o = torch.empty(q.shape, dtype=q.dtype, device=DEV) if o is None else o
    lse = torch.empty(q.shape[0], heads, device=DEV)
    nb = H.hsa_paged_attention_workspace_bytes(q.dtype, q.shape[0], heads, kv, dh, table.shape[1] * page)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if ws is None else ws
    assert ws.numel() >= nb
    H.hsa_paged_attention(d(q), d(held[0]), d(held[1]), d(table), torch.as_tensor(lens, dtype=torch.int32, device=DEV), page,
                          heads, kv, dh, scale, o, ws, k_exp=d(held[2]), v_exp=d(held[3]), lse=lse, **kw)
    return o, lse


PAGED = [
    # lens, page, heads, kv_heads
    ([1], 16, 1, 1),
    ([0, 3, 1], 1, 2, 2),
    ([127, 128, 129, 0], 64, 8, 2),
    ([700], 16, 16, 2),
    ([33, 1025, 2, 300], 100, 5, 1),
    ([511, 4, 90], 32, 17, 1),          # a group over 16 heads
    ([260, 64], 20, 80, 2),
    ([2000, 1, 1, 555], 256, 12, 4),
    ([64, 31, 32, 33] * 5, 7, 3, 3),
]


@pytest.mark.parametrize("lens,page,heads,kv", PAGED, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "e4m3")])
def test_paged(dtype, cache, wide, dh, lens, page, heads, kv):
    """wide: page tables of 5000 rows, whose launch deals tiles of rows to the workgroups and joins the parts."""
    q, k, v, held, table = paged_inputs(sum(lens) + page, dtype, cache, lens, page, heads, kv, dh,
                                        max_pages=5000 // page if wide else None)
    scale = dh ** -0.5
    n_pages = k.shape[0] // page
    o = Guarded(q.shape, T[dtype], 1)
    nb = H.hsa_paged_attention_workspace_bytes(T[dtype], len(lens), heads, kv, dh, table.shape[1] * page)
    ws = Guarded((max(nb, 1),), torch.uint8, 2)
    ws.t.fill_(255)  # NaN in every place that is not written
    _, lse = run_paged(q, held, table, lens, page, heads, kv, dh, scale, o.t, ws.t)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, n_pages, heads, kv, dh, scale)
    check(o.t, lse, want, lw, A, S, dtype, max(lens), dh)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3"), ("f32", "f32")])
@pytest.mark.parametrize("page", [8, 64])
def test_paged_many_sequences_and_one_long(dtype, cache, page):
    lens = [(i * 37) % 200 for i in range(150)] + [9000]
    q, k, v, held, table = paged_inputs(4, dtype, cache, lens, page, 4, 2, 64)
    o, lse = run_paged(q, held, table, lens, page, 4, 2, 64, 0.125)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, k.shape[0] // page, 4, 2, 64, 0.125)
    check(o, lse, want, lw, A, S, dtype, 9000, 64)


@pytest.mark.parametrize("n_seqs,kv,rows", [(n, kv, r) for n, kv in ((1, 1), (16, 4), (13, 5), (32, 4), (43, 3))
                                             for r in (768, 776, 1024, 1032, 2048, 2056)])
def test_paged_table_lengths_where_the_split_changes(n_seqs, kv, rows):
    """Tables just up to and just past each length at which a launch goes over from whole items to dealt tiles,
    in a workspace of exactly the bytes asked for."""
    lens = [rows] + [(i * 613) % (rows + 1) for i in range(1, n_seqs)]
    q, k, v, held, table = paged_inputs(6, "bf16", "bf16", lens, 8, 2 * kv, kv, 64, max_pages=rows // 8)
    nb = H.hsa_paged_attention_workspace_bytes(torch.bfloat16, n_seqs, 2 * kv, kv, 64, rows)
    o, ws = Guarded(q.shape, torch.bfloat16, 1), Guarded((max(nb, 1),), torch.uint8, 2)
    ws.t.fill_(255)
    _, lse = run_paged(q, held, table, lens, 8, 2 * kv, kv, 64, 0.125, o.t, ws.t)
    want, lw, A, S = paged_want(q, k, v, table, lens, 8, k.shape[0] // 8, 2 * kv, kv, 64, 0.125)
    check(o.t, lse, want, lw, A, S, "bf16", rows, 64)
    o.check("o")
    ws.check("workspace")


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,max_pages", [(16, None), (32, None), (48, None), (16, 200), (64, 100)])
def test_paged_bad_pages_are_left_out(cache, page, max_pages):
    lens = [300, 100, 64]
    q, k, v, held, table = paged_inputs(5, "bf16", cache, lens, page, 6, 3, 128, max_pages=max_pages)
    n_pages = k.shape[0] // page
    table[0, 1], table[0, 3], table[1, 0], table[2, :] = -1, n_pages, 2 ** 31 - 1, -2 ** 31
    o, lse = run_paged(q, held, table, lens, page, 6, 3, 128, 0.1)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, n_pages, 6, 3, 128, 0.1)
    check(o, lse, want, lw, A, S, "bf16", 300, 128)
    assert torch.all(o[2] == 0) and torch.all(lse[2] == -math.inf)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")])
@pytest.mark.parametrize("page", [24, 64])
def test_paged_shared_pages_odd_rows_and_long_lengths(dtype, cache, page):
    """Pages shared by sequences; NaN and infinities in rows past a length, in its last page and in pages that no
    sequence names; a length past the table is the table's."""
    heads, kv, dh = 6, 3, 64
    lens = [70, 70, 131]
    q, k, v, held, table = paged_inputs(6, dtype, cache, lens, page, heads, kv, dh, max_pages=-(-131 // page))
    table[1] = table[0]
    n_pages = k.shape[0] // page
    used = torch.zeros(n_pages * page, dtype=torch.bool)
    for s, n in enumerate(lens):
        t = torch.arange(n)
        used[table[s].long()[t // page] * page + t % page] = True
    held = [None if x is None else x.clone() for x in held]
    for x in held[:2]:
        if cache == "e4m3":
            x.view(torch.uint8)[~used] = 0x7f
        else:
            x[~used] = math.nan
            x[(~used).nonzero()[::2, 0]] = math.inf
    o, lse = run_paged(q, held, table, lens, page, heads, kv, dh, 0.2)
    want, lw, A, S = paged_want(q, k, v, table, lens, page, n_pages, heads, kv, dh, 0.2)
    check(o, lse, want, lw, A, S, dtype, 131, dh)
    full = table.shape[1] * page
    table[:] = torch.arange(table.shape[1], dtype=torch.int32) % n_pages
    clean = [k, v] if cache != "e4m3" else None
    if clean:
        o, lse = run_paged(q, (k, v, None, None), table, [2 ** 31 - 1, -5, full], page, heads, kv, dh, 0.2)
        want, lw, A, S = paged_want(q, k, v, table, [full, 0, full], page, n_pages, heads, kv, dh, 0.2)
        check(o, lse, want, lw, A, S, dtype, full, dh)


@pytest.mark.parametrize("max_pages", [0, 3, 300])
def test_paged_without_rows(max_pages):
    """No pages in the table, and no pages in the cache: outputs of zeros."""
    q = torch.ones(2, 256, dtype=torch.bfloat16, device=DEV)
    c = torch.empty(0, 128, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(2, max_pages, dtype=torch.int32)
    o, lse = run_paged(q, (c, c, None, None), table, [5, 0], 16, 2, 1, 128, 0.1)
    assert torch.all(o == 0) and torch.all(lse == -math.inf)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_paged_length_at_the_limit(cache):
    """The longest length the call takes, 2^22 pages of 256 rows, all of them the same page but for the first. Its
    2048 waves add up 2^17 weights in each lane, so sums are off by 2^17 u of themselves at most."""
    q, k, v, held, table = paged_inputs(31, "bf16", cache, [512], 256, 2, 1, 64, spare=0)
    n = 2 ** 30
    table = torch.full((1, n // 256), int(table[0, 1]), dtype=torch.int32).index_fill(1, torch.tensor([0]), int(table[0, 0]))
    o, lse = run_paged(q, held, table, [n], 256, 2, 1, 64, 0.125)
    first, rest = int(table[0, 0]) * 256, int(table[0, 1]) * 256
    for h in range(2):
        # every row of the second page counts 2^22 - 1 times
        s = [(k[r:r + 256].double() @ q[0, h * 64:h * 64 + 64].double()) * 0.125 for r in (first, rest)]
        w = torch.cat([s[0], s[1] + math.log(n // 256 - 1)])
        want = torch.softmax(w, 0) @ torch.cat([v[first:first + 256], v[rest:rest + 256]]).double()
        assert float((o[0, h * 64:h * 64 + 64].cpu().double() - want).abs().max()) < (2.0 ** -7 + 2 ** 18 * U) * float(v.abs().max())
        assert abs(float(lse[0, h]) - float(torch.logsumexp(w, 0))) < 2 ** 17 * U + 1e-5


def test_paged_odd_values_that_are_seen():
    lens, page = [200, 40], 16
    q, k, v, held, table = paged_inputs(7, "bf16", "bf16", lens, page, 2, 1, 64)
    r = int(table[0, 5]) * page + 3
    v[r, 9] = math.inf
    o, _ = run_paged(q, (k, v, None, None), table, lens, page, 2, 1, 64, 0.125)
    assert torch.all(o[0].view(2, 64)[:, 9] == math.inf) and torch.isfinite(o[1]).all()
    k[r, 0] = math.nan
    o, lse = run_paged(q, (k, v, None, None), table, lens, page, 2, 1, 64, 0.125)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all() and torch.isfinite(o[1]).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_offsets_past_32_bits(cache):
    """Rows whose offset in the cache passes 2^31 elements: written, read back and attended to."""
    kv, dh, page = 8, 128, 32
    n_pages = 2 ** 31 // (kv * dh * page) + 40
    n_rows = n_pages * page
    dt = torch.uint8 if cache == "e4m3" else torch.bfloat16
    kc, vc = (torch.empty(n_rows, kv * dh, dtype=dt, device=DEV) for _ in range(2))
    ke = ve = None
    if cache == "e4m3":
        kc, vc = kc.view(F8), vc.view(F8)
        ke, ve = exps(kv, n_rows), exps(kv, n_rows)
    g = _gen(1)
    k, v = _randn(g, 70, kv * dh).bfloat16(), _randn(g, 70, kv * dh).bfloat16()
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32)
    t = torch.arange(70)
    idx = (table[0].long()[t // page] * page + t % page).to(torch.int32).to(DEV)
    H.hsa_cache_store(k.to(DEV), v.to(DEV), idx, 70, kv, kc, vc, ke, ve)
    kb, vb = (torch.empty(70, kv * dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    H.hsa_cache_load(kc, vc, idx, 70, kv, kb, vb, ke, ve)
    if cache == "e4m3":
        for x, b in ((k, kb), (v, vb)):
            codes, ex = quantize64(x, kv)
            assert same(b, (codes.view(70, kv, dh) * torch.pow(2.0, ex.double())[..., None]).view(70, -1))
    else:
        assert same(kb, k) and same(vb, v)
    q = _randn(g, 1, 16 * dh).bfloat16()
    o = torch.empty(1, 16 * dh, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(H.PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    H.hsa_paged_attention(q.to(DEV), kc, vc, table.to(DEV), torch.tensor([70], dtype=torch.int32, device=DEV), page, 16, kv, dh,
                          0.09, o, ws, k_exp=ke, v_exp=ve)
    want = torch.zeros(1, 16 * dh).double()
    A = torch.zeros_like(want)
    for h in range(16):
        c, ck = slice(h * dh, h * dh + dh), slice(h // 2 * dh, h // 2 * dh + dh)
        want[:, c], _, A[:, c], S = attend64(q[:, c], kb.cpu()[:, ck], vb.cpu()[:, ck], torch.ones(1, 70, dtype=torch.bool), 0.09)
    check(o, None, want, None, A, S, "bf16", 70, dh)


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "e4m3")])
def test_prompts_then_tokens(dtype, cache):
    """Prompts attend to themselves and go to their pages; then tokens are generated one at a time, each written to
    its page and attending to all before it. The whole against 64-bit attention over what the caches hold."""
    heads, kv, dh, page = 6, 2, 64, 16
    prompts, steps = [5, 61, 130], 4
    n, scale = len(prompts), 64 ** -0.5
    g = _gen(12)
    width = -(-(max(prompts) + steps) // page)
    table = torch.randperm(n * width, generator=g).view(n, width).to(torch.int32)
    n_rows = n * width * page
    kc, vc = (torch.zeros(n_rows, kv * dh, dtype=torch.uint8, device=DEV).view(F8) if cache == "e4m3" else
              torch.zeros(n_rows, kv * dh, dtype=T[cache], device=DEV) for _ in range(2))
    ke, ve = (exps(kv, n_rows), exps(kv, n_rows)) if cache == "e4m3" else (None, None)
    slot = lambda s, t: int(table[s, t // page]) * page + t % page  # noqa: E731
    full = [[_randn(g, p + steps, w * dh).to(T[dtype]) for w in (heads, kv, kv)] for p in prompts]
    q, k, v = (torch.cat([f[i][:p] for f, p in zip(full, prompts)]) for i in range(3))
    cu = torch.tensor(np.cumsum([0] + prompts), dtype=torch.int32)
    o, _ = run_packed(q, k, v, cu, cu, heads, kv, dh, scale, True)
    want, lw, A, S = packed_want(q, k, v, cu, cu, heads, kv, dh, scale, True)
    check(o, None, want, lw, A, S, dtype, max(prompts), dh)
    idx = torch.tensor([slot(s, t) for s, p in enumerate(prompts) for t in range(p)], dtype=torch.int32, device=DEV)
    H.hsa_cache_store(k.to(DEV), v.to(DEV), idx, len(idx), kv, kc, vc, ke, ve)
    ws = torch.empty(H.PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    for i in range(steps):
        lens = [p + i + 1 for p in prompts]
        q1, k1, v1 = (torch.stack([f[j][p + i] for f, p in zip(full, prompts)]) for j in range(3))
        idx = torch.tensor([slot(s, m - 1) for s, m in enumerate(lens)], dtype=torch.int32, device=DEV)
        H.hsa_cache_store(k1.to(DEV), v1.to(DEV), idx, n, kv, kc, vc, ke, ve)
        o, lse = run_paged(q1, (kc, vc, ke, ve), table, lens, page, heads, kv, dh, scale, ws=ws)
        held = []
        for j in (1, 2):
            rows = torch.zeros(n_rows, kv * dh).double()
            for s, m in enumerate(lens):
                x = full[s][j][:m]
                if cache == "e4m3":
                    codes, ex = quantize64(x, kv)
                    x = (codes.view(m, kv, dh) * torch.pow(2.0, ex.double())[..., None]).view(m, -1)
                rows[[slot(s, t) for t in range(m)]] = x.double()
            held.append(rows)
        want, lw, A, S = paged_want(q1, held[0], held[1], table, lens, page, n * width, heads, kv, dh, scale)
        check(o, lse, want, lw, A, S, dtype, max(lens), dh)


@pytest.mark.parametrize("e4m3", [False, True])
def test_paged_cache_module(e4m3):
    """paged.prefill and paged.decode against one causal pass over the whole sequences: the last rows of a prompt
    that is one longer are what the decoding step gives."""
    heads, kv, dh, page = 8, 2, 128, 32
    prompts = [40, 3, 97]
    g = _gen(14)
    c = paged.PagedCache.allocate(20, page, kv, dh, torch.bfloat16, e4m3=e4m3)
    pages = torch.randperm(20, generator=g).numpy()[:12].reshape(3, 4).astype(np.int32)
    full = [[_randn(g, p + 1, w * dh).bfloat16() for w in (heads, kv, kv)] for p in prompts]
    if e4m3:  # keys and values that 8 bits hold, so that both passes see the same
        for f in full:
            for j in (1, 2):
                codes, ex = quantize64(f[j], kv)
                f[j] = (codes.view(-1, kv, dh) * torch.pow(2.0, ex.double())[..., None]).view(f[j].shape).bfloat16()
    q, k, v = (torch.cat([f[i][:p] for f, p in zip(full, prompts)]).to(DEV) for i in range(3))
    cu = torch.tensor(np.cumsum([0] + prompts), dtype=torch.int32, device=DEV)
    idx = paged.slots(pages, page, np.repeat(np.arange(3), prompts), np.concatenate([np.arange(p) for p in prompts]))
    o = torch.empty_like(q)
    paged.prefill(c, q, k, v, cu, torch.from_numpy(idx).to(DEV), heads, o)
    q1, k1, v1 = (torch.stack([f[i][-1] for f in full]).to(DEV) for i in range(3))
    idx = paged.slots(pages, page, np.arange(3), np.array(prompts))
    o1 = torch.empty_like(q1)
    lens = torch.tensor([p + 1 for p in prompts], dtype=torch.int32, device=DEV)
    paged.decode(c, q1, k1, v1, torch.from_numpy(idx).to(DEV), torch.from_numpy(pages).to(DEV), lens, heads, o1)
    qa, ka, va = (torch.cat([f[i] for f in full]) for i in range(3))
    cu = torch.tensor(np.cumsum([0] + [p + 1 for p in prompts]), dtype=torch.int32)
    want, lw, A, S = packed_want(qa, ka, va, cu, cu, heads, kv, dh, c.scale, True)
    last = cu[1:].long() - 1
    rest = torch.ones(len(qa), dtype=torch.bool)
    rest[last] = False
    check(o, None, want[rest], None, A[rest], S, "bf16", 98, dh)
    check(o1, None, want[last], None, A[last], S, "bf16", 98, dh)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_decode_step_in_a_graph(cache):
    """A captured step (write the new rows, attend) replayed while lengths and rows change, against the eager calls;
    two graphs share one workspace."""
    heads, kv, dh, page, n = 8, 2, 128, 32, 3
    g = _gen(13)
    width = 20
    table = torch.randperm(n * width, generator=g).view(n, width).to(torch.int32)
    n_rows = n * width * page
    base = [_randn(g, n_rows, kv * dh).bfloat16() for _ in range(2)]

    def caches():
        if cache == "bf16":
            return [base[0].to(DEV), base[1].to(DEV), None, None]
        c = [torch.zeros(n_rows, kv * dh, dtype=torch.uint8, device=DEV).view(F8) for _ in range(2)]
        e = [exps(kv, n_rows), exps(kv, n_rows)]
        idx = torch.arange(n_rows, dtype=torch.int32, device=DEV)
        H.hsa_cache_store(base[0].to(DEV), base[1].to(DEV), idx, n_rows, kv, c[0], c[1], e[0], e[1])
        return c + e

    table_d = table.to(DEV)
    ws = torch.empty(H.PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    q, k, v = (torch.zeros(n, w * dh, dtype=torch.bfloat16, device=DEV) for w in (heads, kv, kv))
    lens = torch.ones(n, dtype=torch.int32, device=DEV)
    idx = torch.zeros(n, dtype=torch.int32, device=DEV)

    def step(c, o):
        H.hsa_cache_store(k, v, idx, n, kv, c[0], c[1], c[2], c[3])
        H.hsa_paged_attention(q, c[0], c[1], table_d, lens, page, heads, kv, dh, 0.09, o, ws, k_exp=c[2], v_exp=c[3])

    sets = [caches() for _ in range(3)]
    outs = [torch.empty(n, heads * dh, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for i in range(2):
            step(sets[i], outs[i])
            graph = torch.cuda.CUDAGraph()
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                step(sets[i], outs[i])
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    step(sets[2], outs[2])
    for r, lengths in enumerate(([5, 600, 33], [640, 1, 128], [129, 300, 2])):
        q.copy_(_randn(g, *q.shape).bfloat16())
        k.copy_(_randn(g, *k.shape).bfloat16())
        v.copy_(_randn(g, *v.shape).bfloat16())
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        idx.copy_(torch.tensor([int(table[s, (m - 1) // page]) * page + (m - 1) % page for s, m in enumerate(lengths)],
                               dtype=torch.int32))
        torch.cuda.synchronize()
        graphs[r % 2].replay()
        graphs[1 - r % 2].replay()
        torch.cuda.synchronize()
        step(sets[2], outs[2])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
        outs[0].zero_()
