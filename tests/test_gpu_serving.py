"""GPU tests of what stands around a decoding step: norms of heads with their rotation, and page plans.

Tolerance of the norms, per element (u = 2^-24): the sum of head_dim squares is off by at most (head_dim + 4) u of itself and
the factor by half of that and a few roundings, the two products and the rotation by 4 roundings of
|a cos| + |b sin|, the output by half a step of its type. Plans are whole numbers: equal."""

import math

import pytest
import torch

import test_gpu_seq as S
from gpu_util import Guarded
from paper_2605_06892_amd import hsa_step as H

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def angles(positions, rope_dim, theta=1e4):
    turn = theta ** (-torch.arange(0, rope_dim, 2).double() / rope_dim)
    a = torch.arange(positions).double()[:, None] * turn
    return torch.stack([a.cos(), a.sin()], -1).float()


def norm_want(x, heads, dh, weight, eps, rope, pos, interleaved):
    """The outputs in 64 bits and their bound without the output's rounding: x [n, heads * dh] on the host."""
    n = x.shape[0]
    y = x.double().view(n, heads, dh)
    y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        y = y * weight.double()
    mag = y.abs()
    if rope is not None and rope.shape[1]:
        pairs = rope.shape[1]
        i = torch.arange(pairs)
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        p = torch.arange(n) if pos is None else pos.long()
        ok = (p >= 0) & (p < rope.shape[0])
        cs = rope.double()[p.clamp(0, rope.shape[0] - 1)]
        cos, sin = (torch.where(ok[:, None], cs[..., j], torch.tensor(1.0 - j).double())[:, None] for j in (0, 1))
        a, b = y[..., one].clone(), y[..., two].clone()
        y[..., one], y[..., two] = a * cos - b * sin, a * sin + b * cos
        mag[..., one], mag[..., two] = (a * cos).abs() + (b * sin).abs(), (a * sin).abs() + (b * cos).abs()
    return y.view(n, -1), (dh / 2 + 16) * U * mag.view(n, -1)


def norm_check(got, want, bar, dtype):
    bar = bar + torch.finfo(T[dtype]).eps / 2 * (want.abs() + bar) + 1e-37
    off = (got.cpu().double() - want).abs()
    assert torch.all(off <= bar), f"{float((off / bar).max()):.2f} of the bound"


@pytest.mark.parametrize("n,heads,kv", [(1, 1, 1), (1, 40, 8), (5, 3, 2), (16, 16, 2), (133, 5, 5), (700, 12, 4),
                                        (1501, 40, 7)])  # the last: launches of two heads to a thread, an odd number of them
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rope_dim", [0, 8, 24, 64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_rope(dtype, interleaved, rope_dim, dh, n, heads, kv):
    """Slices of a fused projection, out of place."""
    rope_dim = min(rope_dim, dh)
    g = S._gen(n + dh + rope_dim)
    qkv = (S._randn(g, n, (heads + 2 * kv) * dh) * torch.exp(S._randn(g, n, 1))).to(T[dtype])
    q, k = qkv[:, :heads * dh], qkv[:, heads * dh:(heads + kv) * dh]
    qw, kw = ((1 + 0.3 * S._randn(g, dh)).to(T[dtype]) for _ in range(2))
    rope = angles(300, rope_dim) if rope_dim else None
    pos = torch.randint(-3, 310, (n,), generator=g).to(torch.int32)
    dev = qkv.to(DEV)
    qo, ko = Guarded((n, heads * dh), T[dtype], 1), Guarded((n, kv * dh), T[dtype], 2)
    H.hsa_qk_norm_rope(dev[:, :heads * dh], dev[:, heads * dh:(heads + kv) * dh], heads, kv, dh, qo.t, ko.t, qw.to(DEV), kw.to(DEV),
                       1e-6, None if rope is None else rope.to(DEV), pos.to(DEV), interleaved)
    norm_check(qo.t, *norm_want(q, heads, dh, qw, 1e-6, rope, pos, interleaved), dtype)
    norm_check(ko.t, *norm_want(k, kv, dh, kw, 1e-6, rope, pos, interleaved), dtype)
    assert torch.equal(dev.cpu(), qkv)
    qo.check("q_out")
    ko.check("k_out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n", [1, 3, 77])
def test_norm_rope_in_place(dtype, interleaved, n):
    """Queries and keys turned where they lie, between values that stay: without weights and positions."""
    heads, kv, dh = 6, 2, 128
    qkv = S._randn(S._gen(n), n, (heads + 2 * kv) * dh).to(T[dtype])
    dev = qkv.to(DEV)
    q, k, v = dev.split([heads * dh, kv * dh, kv * dh], 1)
    rope = angles(100, 128)
    H.hsa_qk_norm_rope(q, k, heads, kv, dh, q, k, eps=1e-5, rope=rope.to(DEV), interleaved=interleaved)
    hq, hk, hv = qkv.split([heads * dh, kv * dh, kv * dh], 1)
    norm_check(q, *norm_want(hq, heads, dh, None, 1e-5, rope, None, interleaved), dtype)
    norm_check(k, *norm_want(hk, kv, dh, None, 1e-5, rope, None, interleaved), dtype)
    assert torch.equal(v.cpu(), hv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("side", ["q", "k"])
def test_norm_rope_of_one_alone(dtype, side):
    x = S._randn(S._gen(1), 9, 3 * 64).to(T[dtype])
    out = torch.empty_like(x, device=DEV)
    a = (x.to(DEV), None, 3, 0, 64, out, None) if side == "q" else (None, x.to(DEV), 0, 3, 64, None, out)
    H.hsa_qk_norm_rope(*a)
    norm_check(out, *norm_want(x, 3, 64, None, 1e-6, None, None, False), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_at_the_limits(dtype, interleaved):
    """Magnitudes whose squares fp32 does not hold, zeros, values that are not finite: each head by itself."""
    dh, heads, n = 64, 4, 6
    x = S._randn(S._gen(2), n, heads * dh)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2, :dh] *= 3e37
    x[2, dh:2 * dh] *= 1e-36
    x[3, dh:2 * dh] = 0
    x[4, 5] = math.inf
    x[4, 3 * dh + 1] = math.nan
    x[5] = 3e38
    x = x.to(T[dtype])
    rope, k = angles(10, 64), torch.zeros(n, dh, dtype=T[dtype], device=DEV)
    for eps in (1e-6, 2.0 ** -140, 1e30):
        out, ko = torch.empty_like(x, device=DEV), torch.empty_like(k)
        H.hsa_qk_norm_rope(x.to(DEV), k, heads, 1, dh, out, ko, eps=eps, rope=rope.to(DEV), interleaved=interleaved)
        want, bar = norm_want(x, heads, dh, None, eps, rope, None, interleaved)
        got = out.cpu()
        for h in (0, 3):
            c = slice(h * dh, (h + 1) * dh)
            assert torch.isnan(got[4, c]).any() and torch.equal(torch.isnan(got[4, c]), torch.isnan(want[4, c]))
            want[4, c], got[4, c], bar[4, c] = 0, 0, 0
        norm_check(got, want, bar, dtype)
        assert torch.all(ko == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n", [4, 512])  # the latter in launches of two heads to a thread
def test_norm_rope_keeps_what_is_not_finite_in_its_pair(dtype, interleaved, n):
    """An infinite value makes its channel NaN, and its pair's where that is turned; all others of its head are 0."""
    heads, dh, rope_dim = 64, 128, 64
    x = S._randn(S._gen(3), n, heads, dh).to(T[dtype])
    at = [(0, 2, 70), (0, 3, 127), (1, 0, 5), (2, 1, 9), (3, 63, 40)]
    want = torch.zeros(n, heads, dh, dtype=torch.bool)
    pos = torch.arange(n, dtype=torch.int32)
    pos[2] = -1
    for r, h, c in at:
        x[r, h, c] = math.inf
        want[r, h, c] = True
        if c < rope_dim and r != 2:
            want[r, h, c ^ 1 if interleaved else (c + rope_dim // 2) % rope_dim] = True
    x = x.view(n, -1)
    out = torch.empty(n, heads * dh, dtype=T[dtype], device=DEV)
    H.hsa_qk_norm_rope(x.to(DEV), None, heads, 0, dh, out, None, rope=angles(n, rope_dim).to(DEV), pos=pos.to(DEV),
                       interleaved=interleaved)
    got = out.cpu().view(n, heads, dh)
    assert torch.equal(got.isnan(), want)
    for r, h, _ in at:
        assert torch.all(got[r, h][~want[r, h]] == 0)


def test_norm_rope_turns_as_the_stack_does():
    """A table of one row per token of a grid, the sum of its coordinates' rows of hsa_rope_table."""
    grid, dh, n = (3, 4, 5), 128, 60
    t = H.hsa_rope_table(1e4, dh, grid).view(-1, dh // 2, 2)
    i = torch.arange(n)
    rows = t[i // 20] + t[3 + i // 5 % 4] + t[7 + i % 5]
    x = S._randn(S._gen(1), n, 2 * dh)
    out = torch.empty_like(x, device=DEV)
    H.hsa_qk_norm_rope(x.to(DEV), None, 2, 0, dh, out, None, rope=rows.to(DEV), interleaved=True)
    y = x.double().view(n, 2, dh)
    y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    z = torch.view_as_complex(y.view(n, 2, dh // 2, 2).contiguous())
    turn = torch.zeros(n, dh // 2).double()
    band = 2 * (dh // 6)
    at = 0
    for width, c in ((dh - 2 * band, i // 20), (band, i // 5 % 4), (band, i % 5)):
        j = torch.arange(width // 2).double()
        turn[:, at:at + width // 2] = c.double()[:, None] * 1e4 ** (-2 * j / width)
        at += width // 2
    want = torch.view_as_real(z * torch.polar(torch.ones_like(turn), turn)[:, None]).reshape(n, -1)
    assert float((out.cpu().double() - want).abs().max()) < 200 * U * float(want.abs().max())


def test_norm_rope_refusals_of_the_binding():
    q = torch.ones(4, 256, dtype=torch.bfloat16, device=DEV)
    k = torch.ones(4, 128, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    ok = dict(q=q, k=k, heads=4, kv_heads=2, head_dim=64, q_out=torch.empty_like(q), k_out=torch.empty_like(k), q_weight=w, k_weight=w,
              rope=angles(8, 64).to(DEV), pos=torch.zeros(4, dtype=torch.int32, device=DEV))
    H.hsa_qk_norm_rope(**ok)
    for change in (dict(heads=2), dict(k=None), dict(k_out=None), dict(k=k[:2]), dict(q_weight=w[:32]), dict(rope=ok["rope"][0]),
                   dict(pos=ok["pos"][:3]), dict(q=q.t()), dict(heads=0), dict(q_weight=w.cpu())):
        with pytest.raises(ValueError):
            H.hsa_qk_norm_rope(**{**ok, **change})
    for change in (dict(k=k.float()), dict(q_weight=w.float()), dict(rope=ok["rope"].bfloat16()), dict(pos=ok["pos"].long()),
                   dict(q=q.half()), dict(q=None, k=None)):
        with pytest.raises(TypeError):
            H.hsa_qk_norm_rope(**{**ok, **change})
    for change in (dict(k_out=k[:2].repeat(2, 1), q_out=k.repeat(1, 2), k=k, eps=0.0), dict(q_out=q[:, :], k_out=q[:, :128]),
                   dict(rope=angles(8, 20).to(DEV)), dict(rope=angles(8, 72).to(DEV))):
        with pytest.raises(H.HsaStepError):
            H.hsa_qk_norm_rope(**{**ok, **change})


# ---------------------------------------------------------------- plans


def plan_want(past, fresh, page, table, free, free_at, n_tokens):
    """The definition, one sequence and one token at a time, on the host."""
    table = [list(r) for r in table]
    cap = (len(table[0]) if table else 0) * page
    first, count = (free_at[0] % len(free) if free else 0), max(0, min(free_at[1], len(free)))
    if free and free_at[0] < 0:
        first = (free_at[0] + 2 ** 32) % len(free)
    lacking = 0
    cu, lens, pos, slots = [0], [], [], []
    for s, (p, f) in enumerate(zip(past, fresh)):
        p, f = max(0, min(p, cap)), min(max(f, 0), n_tokens - cu[-1])
        end = min(p + f, cap)
        for i in range(-(-p // page), -(-end // page)):
            if count:
                table[s][i] = free[first]
                first, count = (first + 1) % len(free), count - 1
            else:
                table[s][i] = -1
                lacking += 1
        for t in range(p, p + f):
            pos.append(t)
            row = table[s][t // page] * page + t % page if t < cap and table[s][t // page] >= 0 else -1
            slots.append(row if row < 2 ** 31 else -1)
        cu.append(cu[-1] + f)
        lens.append(end)
    pad = [-1] * (n_tokens - len(pos))
    return table, cu, lens, pos + pad, slots + pad, [first, count, lacking]


def run_plan(past, fresh, page, table, free, free_at, n_tokens, lens_here=False, ring_here=False):
    n, width = len(past), len(table[0]) if table else 0
    d = lambda x, *s: torch.tensor(x, dtype=torch.int32, device=DEV).view(*s) if s else torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    g = {name: Guarded((size,), torch.int32, i) for i, (name, size) in enumerate(
        [("cu", n + 1), ("lens", max(n, 1)), ("pos", max(n_tokens, 1)), ("slots", max(n_tokens, 1)), ("next", 3), ("table", max(n * width, 1))])}
    for x in g.values():
        x.t.fill_(77)
    t = g["table"].t[:n * width].view(n, width)
    t.copy_(d([x for r in table for x in r], n, width) if n * width else t)
    past_d, at_d = d(past), d(list(free_at) + [55])
    lens, nxt = past_d if lens_here else g["lens"].t[:n], at_d if ring_here else g["next"].t
    H.hsa_page_plan(past_d, d(fresh), page, t, d(free), at_d, g["cu"].t, lens, g["pos"].t[:n_tokens], g["slots"].t[:n_tokens], nxt)
    for name, x in g.items():
        x.check(name)
    return [x.tolist() for x in (t, g["cu"].t, lens, g["pos"].t[:n_tokens], g["slots"].t[:n_tokens], nxt)]


def plan_inputs(seed, past, page, width, n_free, spare=0):
    import random
    r = random.Random(seed)
    have = [min(width, -(-max(p, 0) // page)) for p in past]
    pages = list(range(sum(have) + n_free + spare))
    r.shuffle(pages)
    table, at = [], 0
    for h in have:
        table.append(pages[at:at + h] + [-9] * (width - h))
        at += h
    return table, pages[at:at + n_free]


PLANS = [
    # past, fresh, page, width, n_free, free_at, tokens beyond the fresh ones
    ([0], [1], 16, 3, 2, (0, 2), 0),
    ([5], [0], 16, 3, 2, (1, 2), 3),
    ([15, 16, 17, 0], [1, 1, 1, 1], 16, 4, 9, (7, 9), 0),
    ([0, 0, 0], [33, 0, 64], 32, 3, 8, (6, 5), 5),
    ([100, 3, 0, 7], [50, 200, 1, 0], 7, 40, 60, (0, 60), 1),
    ([10, 10, 10], [40, 40, 40], 16, 8, 5, (3, 4), 0),               # fewer pages than needed
    ([10, 0], [0, 0], 16, 2, 0, (0, 0), 2),                          # none at all
    ([40, 60, 64], [20, 20, 20], 16, 4, 9, (2, 9), 0),               # past the table's width
    ([-4, 1000, 3], [5, 2, -6], 8, 4, 9, (-1, 100), 2),              # lengths and a ring out of range
    ([0] * 7, [1] * 7, 1, 2, 9, (8, 9), 0),
    ([2, 3], [5, 5], 100, 0, 4, (0, 4), 1),                          # no table
    ([i * 7 % 90 for i in range(1500)], [i * 13 % 40 for i in range(1500)], 20, 7, 5000, (4000, 5000), 17),
    ([i * 7 % 90 for i in range(4097)], [1] * 4097, 64, 2, 3000, (100, 3000), 0),
    ([0, 0, 0], [5000, 1, 9000], 16, 563, 1200, (1100, 1200), 0),
]


@pytest.mark.parametrize("past,fresh,page,width,n_free,at,pad", PLANS, ids=range(len(PLANS)))
@pytest.mark.parametrize("here", [(False, False), (True, True), (True, False), (False, True)], ids=["apart", "here", "lens", "ring"])
def test_plan(past, fresh, page, width, n_free, at, pad, here):
    table, free = plan_inputs(len(past) + page, past, page, width, n_free)
    n_tokens = sum(max(f, 0) for f in fresh) + pad
    assert run_plan(past, fresh, page, table, free, at, n_tokens, *here) == list(plan_want(past, fresh, page, table, free, at, n_tokens))


@pytest.mark.parametrize("n_tokens", [0, 1, 63, 64, 150])
@pytest.mark.parametrize("here", [False, True])
def test_plan_of_fewer_tokens_than_fresh(n_tokens, here):
    """What is beyond the capacity does not count, garbage that would sum past 32 bits among it."""
    past, fresh = [3, 60, 0, 9, 1], [60, 70, 2 ** 31 - 1, 2 ** 31 - 1, 5]
    table, free = plan_inputs(1, past, 16, 12, 30)
    assert run_plan(past, fresh, 16, table, free, (3, 30), n_tokens, here, here) == \
        list(plan_want(past, fresh, 16, table, free, (3, 30), n_tokens))


def test_plan_of_nothing():
    assert run_plan([], [], 16, [], [4, 5], (1, 2), 0)[1:] == [[0], [], [], [], [1, 2, 0]]
    assert run_plan([], [], 16, [], [], (9, 2), 3)[1:] == [[0], [], [-1] * 3, [-1] * 3, [0, 0, 0]]


def test_plan_rows_past_int32():
    """Page numbers whose rows do not fit int32, and negative ones, give no slot."""
    table = [[2 ** 28, 2 ** 27 - 1, -1], [2 ** 31 - 1, -2 ** 31, 5]]
    past, fresh = [0, 0], [48, 48]
    got = run_plan([16, 16], [40, 0], 16, table, [2 ** 30, 7], (0, 2), 40)
    assert got == list(plan_want([16, 16], [40, 0], 16, table, [2 ** 30, 7], (0, 2), 40))
    assert got[4][:16] == [-1] * 16 and got[4][16] == 7 * 16
    got = run_plan([40, 33], [4, 4], 16, table, [1], (0, 1), 8)
    assert got == list(plan_want([40, 33], [4, 4], 16, table, [1], (0, 1), 8)) and got[4][:4] == [-1] * 4
    assert past and fresh


def test_plan_steps_in_a_graph():
    """A captured step that goes on from its own lengths and ring, replayed with other fresh counts each time."""
    page, width, n_tokens = 8, 12, 32
    past, (table, free) = [3, 0, 17, 8], plan_inputs(5, [3, 0, 17, 8], 8, 12, 25)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    lens, fresh, t, ring, at = i32(past), i32([0] * 4), i32(table), i32(free), i32([20, 25, 0])
    cu, pos, slots = torch.empty(5, dtype=torch.int32, device=DEV), *(torch.empty(n_tokens, dtype=torch.int32, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        H.hsa_page_plan(lens, fresh, page, t, ring, at, cu, lens, pos, slots, at)
    state = [20, 25]
    for f in ([1, 1, 1, 1], [5, 9, 0, 8], [0, 0, 0, 0], [30, 1, 1, 9], [20, 20, 20, 20]):
        fresh.copy_(i32(f))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        table, cu_w, past, pos_w, slots_w, state = plan_want(past, f, page, table, free, state[:2], n_tokens)
        assert [x.tolist() for x in (t, cu, lens, pos, slots, at)] == [table, cu_w, past, pos_w, slots_w, state]


def test_plan_refusals_of_the_binding():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    ok = dict(past=i(3), fresh=i(3), page_size=16, page_table=i(3, 4), free_pages=i(9), free_at=i(3), cu=i(4), kv_lens=i(3), pos=i(8),
              slots=i(8), free_next=i(3))
    H.hsa_page_plan(**ok)
    for change in (dict(fresh=i(2)), dict(cu=i(3)), dict(page_table=i(12)), dict(page_table=i(2, 4)), dict(pos=i(7)), dict(free_at=i(2)),
                   dict(page_table=i(4, 3).t()), dict(past=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            H.hsa_page_plan(**{**ok, **change})
    for change in (dict(past=i(3).long()), dict(slots=i(8).float())):
        with pytest.raises(TypeError):
            H.hsa_page_plan(**{**ok, **change})
    for change in (dict(page_size=0), dict(slots=ok["pos"]), dict(kv_lens=ok["fresh"]), dict(free_next=ok["past"])):
        with pytest.raises(H.HsaStepError):
            H.hsa_page_plan(**{**ok, **change})
