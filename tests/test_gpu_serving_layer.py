"""GPU tests of paged.py's layer with weights in 4 bits over a cache in 4 bits: plan, projections, norms, rotation, store and
attention as they are used together. Every tensor is held to its definition in 64 bits on the tensors that
went into it, with the bounds of test_gpu_four_bit.py, test_gpu_serving.py and test_gpu_seq.py."""

import pytest
import torch

import test_gpu_four_bit as F
import test_gpu_seq as S
import test_gpu_serving as N
from gpu_util import Guarded
from paper_2605_06892_amd import hsa_step as H
from paper_2605_06892_amd import paged

pytestmark = pytest.mark.gpu

DEV = "cuda"
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def layer(g, dtype, d, heads, kv, dh, n_tokens):
    w_qkv, w_out = (S._randn(g, n, k).to(T[dtype]).to(DEV) * k ** -0.5 for n, k in (((heads + 2 * kv) * dh, d), (d, heads * dh)))
    q_norm, k_norm = ((1 + 0.2 * S._randn(g, dh)).to(T[dtype]).to(DEV) for _ in range(2))
    return paged.Layer4.allocate(w_qkv, w_out, heads, kv, dh, n_tokens, q_norm, k_norm)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh,page", [(6, 2, 64, 16), (5, 5, 128, 32), (8, 1, 64, 20)])
def test_prompts_then_tokens(dtype, heads, kv, dh, page):
    d, prompts, steps = 192, [5, 61, 130], 3
    n, g = len(prompts), S._gen(heads)
    total = sum(prompts)
    width = -(-(max(prompts) + steps) // page)
    n_pages = n * width + 2
    lay = layer(g, dtype, d, heads, kv, dh, total)
    c = paged.PagedCache.allocate(n_pages, page, kv, dh, T[dtype], e2m1=True)
    pool = paged.PagePool.allocate(n_pages, page, n, width, total)
    rope = N.angles(300, dh).to(DEV)
    lens = [0] * n
    for step in range(steps + 1):
        fresh = prompts if step == 0 else [1] * n
        tokens = sum(fresh)
        before, free, at = pool.page_table.tolist(), pool.free.tolist(), pool.free_at.tolist()
        pool.plan(i32(fresh))
        want = N.plan_want(lens, fresh, page, before, free, at[:2], total)
        assert [x.tolist() for x in (pool.page_table, pool.cu, pool.lens, pool.pos, pool.slots, pool.free_at)] == list(want)
        lens = [a + b for a, b in zip(lens, fresh)]
        x = S._randn(g, tokens, d).to(T[dtype]).to(DEV)
        y = torch.empty_like(x)
        lay.step(x, c, pool, rope, y, prompts=step == 0)
        # the projection again, for the layer's own was normed where it lies
        scale, qkv = torch.empty(tokens, device=DEV), torch.empty(tokens, (heads + 2 * kv) * dh, dtype=T[dtype], device=DEV)
        H.hsa_row_rms_scale(x, tokens, scale)
        H.hsa_linear_w4(x, tokens, *lay.w_qkv, qkv, row_scale=scale)
        F.linear_check(qkv, x.cpu(), *(t.cpu() for t in lay.w_qkv), dtype, scale.cpu())
        a, b = heads * dh, (heads + kv) * dh
        q, k, v = (t.cpu() for t in lay.qkv[:tokens].split([a, kv * dh, kv * dh], 1))
        pos = pool.pos[:tokens].cpu()
        N.norm_check(q, *N.norm_want(qkv[:, :a].cpu(), heads, dh, lay.q_norm.cpu(), 1e-6, rope.cpu(), pos, False), dtype)
        N.norm_check(k, *N.norm_want(qkv[:, a:b].cpu(), kv, dh, lay.k_norm.cpu(), 1e-6, rope.cpu(), pos, False), dtype)
        assert torch.equal(v, qkv[:, b:].cpu())
        slots = pool.slots[:tokens].cpu().long()
        for t, codes, ex in ((k, c.k, c.k_exp), (v, c.v, c.v_exp)):
            _, packed, e = F.quantize4(t)
            assert torch.equal(codes.cpu()[slots], packed) and torch.equal(ex.cpu()[slots], e)
        o = lay.o[:tokens]
        if step == 0:
            cu = pool.cu.cpu()
            want, _, A, Sm = S.packed_want(q, k, v, cu, cu, heads, kv, dh, dh ** -0.5, True)
        else:
            kc, vc = F.values4(c.k.cpu(), c.k_exp.cpu()), F.values4(c.v.cpu(), c.v_exp.cpu())
            want, _, A, Sm = S.paged_want(q, kc, vc, pool.page_table.cpu(), lens, page, n_pages, heads, kv, dh, dh ** -0.5)
        S.check(o, None, want, None, A, Sm, dtype, max(lens), dh)
        F.linear_check(y, o.cpu(), *(t.cpu() for t in lay.w_out), dtype, residual=x.cpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decoding_in_a_graph(dtype):
    """Captured steps of two layers that share a workspace, a pool and their hidden rows, replayed while the lengths grow past
    pages, against eager steps of a pool and caches of their own."""
    heads, kv, dh, page, d, n, width = 4, 2, 128, 8, 128, 5, 4
    g = S._gen(9)
    layers = [layer(g, dtype, d, heads, kv, dh, n) for _ in range(2)]
    rope = N.angles(64, dh).to(DEV)

    def world():
        a = paged.PagedCache.allocate(n * width, page, kv, dh, T[dtype], e2m1=True)
        b = paged.PagedCache.allocate(n * width, page, kv, dh, T[dtype], e2m1=True, workspace=a.workspace)
        return a, b, paged.PagePool.allocate(n * width, page, n, width, n), torch.empty(n, d, dtype=T[dtype], device=DEV)

    one = i32([1] * n)
    worlds = [world() for _ in range(2)]

    def step(a, b, pool, h):
        pool.plan(one)
        layers[0].step(h, a, pool, rope, h)
        layers[1].step(h, b, pool, rope, h)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*worlds[0])
    for i in range(20):
        x = S._randn(g, n, d).to(T[dtype]).to(DEV)
        for w in worlds:
            w[3].copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(*worlds[1])
        torch.cuda.synchronize()
        (_, _, p, h), (_, _, q, want) = worlds
        assert torch.isfinite(want.float()).all() and torch.equal(h, want)
        assert torch.equal(p.page_table, q.page_table) and p.lens.tolist() == q.lens.tolist() == [i + 1] * n
        assert p.free_at.tolist() == q.free_at.tolist() == [n * (-(-(i + 1) // page)) % (n * width), n * width - n * (-(-(i + 1) // page)), 0]


def test_sequences_come_and_go():
    """A finished sequence's pages serve another's, and a pool that runs out says so."""
    pool = paged.PagePool.allocate(6, 8, 3, 5, 40)
    pool.plan(i32([17, 8, 15]))  # three, one and two pages: all
    assert pool.free_at.tolist()[1:] == [0, 0] and int((pool.slots >= 0).sum()) == 40
    pool.plan(i32([0, 1, 1]))    # one page is lacking
    assert pool.free_at.tolist()[1:] == [0, 1] and pool.slots[:3].tolist()[0] == -1 and pool.lens.tolist() == [17, 9, 16]
    first = pool.page_table[0, :3].tolist()
    pool.release(0)
    pool.release(1)
    assert pool.lens.tolist() == [0, 0, 16] and int(pool.free_at[1]) == 4
    pool.plan(i32([24, 0, 1]))
    assert pool.free_at.tolist()[1:] == [0, 0] and torch.all(pool.slots[:25] >= 0)
    used = [x for r in pool.page_table.tolist() for x in r if x >= 0]
    assert len(set(used)) == len(used) == 6 and set(first) <= set(used)


def test_step_of_too_many_tokens():
    """Refused before anything is enqueued: what lies behind the layer's row scales stays, and so do the caches."""
    lay = layer(S._gen(3), "bf16", 128, 4, 2, 64, 4)
    guarded = Guarded((4,), torch.float32, 5)
    lay.scale = guarded.t
    lay.scale.fill_(7)
    c = paged.PagedCache.allocate(16, 8, 2, 64, torch.bfloat16, e2m1=True)
    c.k.fill_(3)
    pool = paged.PagePool.allocate(16, 8, 5, 3, 9)
    pool.plan(i32([1] * 5))
    for n, prompts in ((5, False), (9, True), (4, False)):
        x = torch.ones(n, 128, dtype=torch.bfloat16, device=DEV)
        with pytest.raises(ValueError):
            lay.step(x, c, pool, None, x, prompts=prompts)
        with pytest.raises(ValueError):
            H.hsa_row_rms_scale(x, n + 1, torch.empty(n + 1, device=DEV))
        if n > 4:
            with pytest.raises(ValueError):
                H.hsa_row_rms_scale(x, n, lay.scale)
    torch.cuda.synchronize()
    guarded.check("scale")
    assert torch.all(lay.scale == 7) and torch.all(c.k == 3)


def test_a_page_that_was_lacking_is_reported_and_made_good():
    """Run out, free another sequence's page, plan one more token into the page that was lacking."""
    pool = paged.PagePool.allocate(2, 8, 2, 3, 8)
    pool.plan(i32([4, 4]))
    pool.plan(i32([4, 4]))
    assert pool.lacked.tolist() == [0] and pool.free_at.tolist()[1:] == [0, 0]
    pool.plan(i32([0, 1]))
    assert pool.lacked.tolist() == [1] and pool.free_at.tolist()[1:] == [0, 1] and pool.slots[:1].tolist() == [-1]
    pool.release(0)
    pool.plan(i32([0, 1]))
    assert pool.lacked.tolist() == [1] and pool.slots[:1].tolist() == [-1] and pool.lens.tolist() == [0, 10]
    assert pool.resume(0) == 0 and pool.resume(1) == 2 and pool.lens.tolist() == [0, 8]
    pool.lacked.zero_()
    pool.plan(i32([0, 2]))
    page = int(pool.page_table[1, 1])
    assert page >= 0 and pool.slots[:2].tolist() == [page * 8, page * 8 + 1] and pool.pos[:2].tolist() == [8, 9]
    assert pool.lacked.tolist() == [0] and pool.lens.tolist() == [0, 10] and pool.free_at.tolist()[1:] == [0, 0]


def test_lacking_pages_are_counted_over_replayed_steps():
    page, n, width, pages = 4, 5, 9, 22
    pool, one = paged.PagePool.allocate(pages, page, n, width, n), i32([1] * n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.plan(one)
    for i in range(30):
        graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
            assert pool.lacked.tolist() == [max(0, n * -(-(i + 1) // page) - pages)]
    assert pool.lacked.tolist() == [n * -(-30 // page) - pages] and pool.free_at.tolist()[1] == 0
    assert [pool.resume(s) for s in range(n)] == [30 - 4 * 5 if s < 2 else 30 - 4 * 4 for s in range(n)]
    assert pool.lens.tolist() == [20, 20, 16, 16, 16]
