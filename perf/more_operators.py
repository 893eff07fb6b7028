"""Performance cases of a serving step in 4 bits: weights and caches in e2m1 codes, and what stands between them.

Five operators of one path. A group is 32 consecutive values: 16 bytes of e2m1 codes, the even one in the low half of each
byte, and one signed power-of-two exponent.

  linear  `hsa_linear_w4`: rows times weights in 4 bits, with the row map's epilogue
  norm    `hsa_qk_norm_rope`: RMS norms of every head of queries and keys, and their rotation by position
  plan    `hsa_page_plan`: pages, cache rows, positions and offsets of fresh tokens, from the sequences' lengths
  swap    `hsa_cache_store`, `hsa_cache_load`: rows into a 4-bit cache and back
  paged   `hsa_paged_attention`: one query per sequence over pages of a 4-bit cache

`own` says which side `run` takes: the plain form in elementary torch operations, or the library's calls.
Widths and token counts are those of `synth.WORKLOADS` or generic ones.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32
EXP_MIN, EXP_MAX = -125, 125  # exponents of a group of finite values
EPS = 1e-6
THETA = 1e6
PAGED_WORKSPACE = 32 << 20  # HSA_STEP_PAGED_WORKSPACE_BYTES: enough for any call, kept by a serving loop


def listed():
    return [
        # the next token of one conversation through a small model's first FFN product, its norm and GELU: latency
        {"name": "linear_token", "kind": "linear", "dtype": "bf16", "out": "bf16", "rows": 1, "d_in": 1536, "d_out": 8960,
         "scaled": True, "gelu": True, "residual": False},
        # a verification run's second FFN product in fp32 with the residual, a few sequences, an odd width
        {"name": "linear_f32", "kind": "linear", "dtype": "f32", "out": "f32", "rows": 5, "d_in": 8960, "d_out": 1537,
         "scaled": False, "gelu": False, "residual": True},
        # a batch's logits over a vocabulary: the weights' bytes bound it
        {"name": "linear_logits", "kind": "linear", "dtype": "bf16", "out": "f32", "rows": 16, "d_in": 8192, "d_out": 32768,
         "scaled": True, "gelu": False, "residual": False},
        # one decoding step of 16 sequences: latency
        {"name": "norm_step", "kind": "norm", "dtype": "bf16", "rows": 16, "heads": 40, "kv_heads": 8, "head_dim": 128,
         "rope_dim": 128, "interleaved": False, "positions": 8192},
        # the active quarter of a 480p clip's tokens at the large model's width
        {"name": "norm_480p", "kind": "norm", "dtype": "bf16", "rows": 8190, "heads": 40, "kv_heads": 40, "head_dim": 128,
         "rope_dim": 128, "interleaved": True, "positions": 32760},
        # one new token for each of a serving batch's sequences, a page now and then
        {"name": "plan_step", "kind": "plan", "seqs": 48, "past_from": 201, "past_to": 8009, "fresh_from": 1, "fresh_to": 1,
         "page": 64, "pad": 16},
        # a thousand prompts at once, in small pages, some of them continued
        {"name": "plan_prompts", "kind": "plan", "seqs": 1000, "past_from": 0, "past_to": 1500, "fresh_from": 1,
         "fresh_to": 2047, "page": 16, "pad": 0},
        # a suspended sample's active rows in 4 bits and back, fp32 and odd
        {"name": "swap_ragged_f32", "kind": "swap", "dtype": "f32", "rows": 777, "cache_rows": 1024, "kv_heads": 5,
         "head_dim": 64},
        # a whole layer cache of a 480p clip suspended in 4 bits and resumed
        {"name": "swap_480p", "kind": "swap", "dtype": "bf16", "rows": 32760, "cache_rows": 32760, "kv_heads": 12,
         "head_dim": 128},
        # one conversation's next token: latency
        {"name": "paged_one", "kind": "paged", "dtype": "bf16", "seqs": 1, "shortest": 700, "longest": 700, "page": 16,
         "heads": 16, "kv_heads": 2, "head_dim": 64},
        # a serving batch's next tokens, contexts of very different lengths
        {"name": "paged_batch", "kind": "paged", "dtype": "bf16", "seqs": 48, "shortest": 201, "longest": 8009, "page": 64,
         "heads": 32, "kv_heads": 8, "head_dim": 128},
        # a few very long contexts: the cache's bytes bound it
        {"name": "paged_long", "kind": "paged", "dtype": "bf16", "seqs": 4, "shortest": 30011, "longest": 131072,
         "page": 128, "heads": 40, "kv_heads": 8, "head_dim": 128},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "norm", "plan", "swap", "paged"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dh = rng.choice([64, 128])
    es = 2 if dtype == "bf16" else 4
    if kind == "linear":
        rows = _log(rng, 1, 64)
        d_in = GROUP * _log(rng, 2, 512)
        # the products of the largest listed case at most; fp32 ones run at a fraction of the rate
        most = min(8192 * 32768, 16 * 8192 * 32768 // (rows * (1 if dtype == "bf16" else 8)))
        d_out = _log(rng, 1, max(1, min(32768, most // d_in)))
        out = "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"])
        gelu = out == dtype and rng.random() < 0.3
        return {"kind": kind, "dtype": dtype, "out": out, "rows": rows, "d_in": d_in, "d_out": d_out,
                "scaled": rng.random() < 0.5, "gelu": gelu, "residual": out == dtype and not gelu and rng.random() < 0.5}
    if kind == "norm":
        kv, group = rng.randint(1, 16), rng.choice([1, 1, 2, 3, 4, 5, 7, 8])
        heads = min(kv * group, 64 // kv * kv)
        positions = _log(rng, 64, 131072)
        rows = _log(rng, 1, max(1, min(32760, 8190 * 80 * 128 * 2 // ((heads + kv) * dh * es))))
        return {"kind": kind, "dtype": dtype, "rows": rows, "heads": heads, "kv_heads": kv, "head_dim": dh,
                "rope_dim": rng.choice([dh, dh, dh, dh // 2, 24, 40, 0]), "interleaved": rng.random() < 0.5,
                "positions": positions}
    if kind == "plan":
        seqs = _log(rng, 1, 2000)
        most = min(8192, 1000 * 2047 // seqs)
        fresh_to = rng.choice([1, _log(rng, 1, most)])
        past_to = _log(rng, 1, 8192)
        return {"kind": kind, "seqs": seqs, "past_from": rng.choice([0, _log(rng, 1, past_to)]), "past_to": past_to,
                "fresh_from": rng.randint(0, fresh_to) if fresh_to > 1 else 1, "fresh_to": fresh_to,
                "page": rng.choice([1, 8, 16, 20, 32, 64, 100, 128, 256]), "pad": rng.choice([0, _log(rng, 1, 64)])}
    kv = rng.randint(1, 16)
    if kind == "swap":
        rows = _log(rng, 1, max(1, min(32760, 32760 * 12 * 128 * 2 // (kv * dh * es))))
        return {"kind": kind, "dtype": dtype, "rows": rows, "cache_rows": rows + _log(rng, 1, 4096), "kv_heads": kv,
                "head_dim": dh}
    group = rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8, 16])
    if kv * group > 64:
        kv = 64 // group
    seqs = _log(rng, 1, 128)
    most = 290000 * 8 * 128 // (seqs * kv * dh * (1 if dtype == "bf16" else 2))
    longest = _log(rng, 1, min(131072, most))
    return {"kind": kind, "dtype": dtype, "seqs": seqs, "shortest": _log(rng, 1, longest), "longest": longest,
            "page": rng.choice([1, 8, 16, 20, 32, 64, 100, 128, 256]), "heads": kv * group, "kv_heads": kv, "head_dim": dh}


def spread(n, lo, hi):
    """n lengths from lo to hi, in equal ratios from 1 on, in a mixed order."""
    if n == 1:
        return [hi]
    a, b = max(lo, 1), max(hi, 1)
    up = [lo if i == 0 else int(round(a * (b / a) ** (i / (n - 1)))) for i in range(n)]
    step = next(s for s in range(n // 2 + 1, 2 * n + 2) if math.gcd(s, n) == 1)
    return [up[(i * step) % n] for i in range(n)]


def _plan_lengths(case):
    past = spread(case["seqs"], case["past_from"], case["past_to"])
    fresh = spread(case["seqs"], case["fresh_from"], case["fresh_to"])
    return past, fresh[1:] + fresh[:1]


def _lut():
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)


def _pow2(e):
    """2^e in fp32, for exponents of normal numbers."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantize(x):
    """e2m1 codes of the last dimension's groups, two to a byte, and the int8 exponent of each: x is codes * 2^exponent, the
    exponent the smallest with which the greatest magnitude is at most 6."""
    y = x.float().view(*x.shape[:-1], -1, GROUP)
    frac, ex = torch.frexp(y.abs().amax(-1))
    ex = torch.where(frac <= 0.75, ex - 3, ex - 2).clamp(EXP_MIN, EXP_MAX)
    y = (y * _pow2(-ex)[..., None]).clamp(-6.0, 6.0)
    mag = y.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    mag = torch.round(mag / step) * step
    code = torch.where(mag < 2, 2 * mag, torch.where(mag < 4, mag + 2, mag / 2 + 4)).to(torch.uint8)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).view(*x.shape)
    return code[..., 0::2] + 16 * code[..., 1::2], ex.to(torch.int8)


def _values(codes, ex):
    """fp32 values of rows of codes."""
    y = torch.stack([codes & 15, codes >> 4], -1).view(*codes.shape[:-1], -1)
    y = _lut()[y.int()].view(*ex.shape, GROUP)
    return (y * _pow2(ex)[..., None]).view(*codes.shape[:-1], -1)


def _keys(k, kv_heads):
    """Keys have a few channels far larger than the others, the same ones in every row."""
    k.view(k.shape[0], kv_heads, -1)[..., 5::32] *= 6.0
    return k


def _rows_in_turns(f, n, width):
    """f(rows) of n rows of `width` values, a limited number at a time, joined."""
    turn = max(1, (1 << 26) // width)
    parts = [f(min(turn, n - a)) for a in range(0, n, turn)]
    return tuple(torch.cat(x) for x in zip(*parts))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def randn(*s):
        return torch.randn(*s, generator=g, device=DEV)

    st = {"case": case}
    if case["kind"] == "linear":
        t, to, rows, d_in, d_out = TYPES[case["dtype"]], TYPES[case["out"]], case["rows"], case["d_in"], case["d_out"]
        x = randn(rows, d_in)
        x[:, 7::64] *= 8.0  # a few channels of the residual stream are far larger than the others
        st["x"] = x.to(t)
        st["w"], st["w_exp"] = _rows_in_turns(lambda n: _quantize(randn(n, d_in) * d_in ** -0.5), d_out, d_in)
        st["scale"] = 1 / (st["x"].float().square().mean(1) + EPS).sqrt() if case["scaled"] else None
        st["residual"] = randn(rows, d_out).to(to) if case["residual"] else None
        st["y"] = torch.empty(rows, d_out, dtype=to, device=DEV)
        return st
    if case["kind"] == "plan":
        past, fresh = _plan_lengths(case)
        page, pad = case["page"], case["pad"]
        have = [-(-p // page) for p in past]
        need = [-(-(p + f) // page) - h for p, f, h in zip(past, fresh, have)]
        spare = 5 + sum(need) // 4
        order = torch.randperm(sum(have) + sum(need) + spare, generator=g, device=DEV).to(torch.int32)
        st["free"] = order[sum(have):].contiguous()  # a ring: from an entry in its middle on, all of it
        st["page_table"] = torch.full((len(past), max(h + n for h, n in zip(have, need)) + 2), -1, dtype=torch.int32, device=DEV)
        rank = torch.arange(st["page_table"].shape[1], device=DEV)
        held = rank < torch.tensor(have, device=DEV)[:, None]
        st["page_table"][held] = order[:sum(have)]
        ints = torch.tensor([past, fresh], dtype=torch.int32, device=DEV)
        st["past"], st["fresh"] = ints[0].contiguous(), ints[1].contiguous()
        n_free = st["free"].numel()
        st["free_at"] = torch.tensor([n_free * 2 // 3, n_free, 0], dtype=torch.int32, device=DEV)
        st["tokens"] = sum(fresh) + pad
        st["cu"] = torch.empty(len(past) + 1, dtype=torch.int32, device=DEV)
        st["kv_lens"] = torch.empty(len(past), dtype=torch.int32, device=DEV)
        st["pos"], st["slots"] = (torch.empty(st["tokens"], dtype=torch.int32, device=DEV) for _ in range(2))
        st["free_next"] = torch.empty(3, dtype=torch.int32, device=DEV)
        return st
    t, kv, dh = TYPES[case["dtype"]], case["kv_heads"], case["head_dim"]
    d = kv * dh
    if case["kind"] == "norm":
        n, heads, rot = case["rows"], case["heads"], case["rope_dim"]
        qkv = randn(n, heads * dh + 2 * d) * 3.0  # the fused projection's output: queries, keys, values
        qkv[:, heads * dh:heads * dh + d] = _keys(qkv[:, heads * dh:heads * dh + d].contiguous(), kv)
        st["q"], st["k"], _ = qkv.to(t).split([heads * dh, d, d], dim=1)
        st["q_weight"], st["k_weight"] = ((1 + 0.3 * randn(dh)).to(t) for _ in range(2))
        st["pos"] = torch.randint(case["positions"], (n,), generator=g, device=DEV, dtype=torch.int32)
        st["rope"] = None
        if rot:
            turn = THETA ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
            angle = torch.arange(case["positions"], device=DEV, dtype=torch.float64)[:, None] * turn
            st["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        st["q_out"] = torch.empty(n, heads * dh, dtype=t, device=DEV)
        st["k_out"] = torch.empty(n, d, dtype=t, device=DEV)
        return st
    if case["kind"] == "swap":
        n, rows = case["rows"], case["cache_rows"]
        st["idx"] = torch.randperm(rows, generator=g, device=DEV)[:n].to(torch.int32)
        kvs = randn(n, 2 * d)  # the fused projection's output: keys beside values
        kvs[:, :d] = _keys(kvs[:, :d].contiguous(), kv)
        st["k"], st["v"] = kvs.to(t).split([d, d], dim=1)
        st["k_cache"], st["k_exp"] = _quantize(_keys(randn(rows, d), kv))
        st["v_cache"], st["v_exp"] = _quantize(randn(rows, d))
        st["k_back"], st["v_back"] = (torch.empty(n, d, dtype=t, device=DEV) for _ in range(2))
        return st
    lens, page, heads = spread(case["seqs"], case["shortest"], case["longest"]), case["page"], case["heads"]
    n = len(lens)
    need = torch.tensor([-(-x // page) for x in lens], device=DEV)
    pages = int(need.sum()) + 3
    width = int(need.max())
    st["page_table"] = torch.zeros(n, width, dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV) < need[:, None]
    st["page_table"][held] = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)[:pages - 3]
    st["kv_lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    rows = pages * page
    st["k_cache"], st["k_exp"] = _rows_in_turns(lambda m: _quantize(_keys(randn(m, d), kv)), rows, d)
    st["v_cache"], st["v_exp"] = _rows_in_turns(lambda m: _quantize(randn(m, d)), rows, d)
    st["q"] = randn(n, heads * dh).to(t)
    st["o"] = torch.empty(n, heads * dh, dtype=t, device=DEV)
    st["lse"] = torch.empty(n, heads, device=DEV)
    st["workspace"] = torch.empty(PAGED_WORKSPACE, dtype=torch.uint8, device=DEV)
    return st


def _own(st):
    from paper_2605_06892_amd import hsa_step as H

    c = st["case"]
    if c["kind"] == "linear":
        H.hsa_linear_w4(st["x"], c["rows"], st["w"], st["w_exp"], st["y"], residual=st["residual"], row_scale=st["scale"],
                        gelu=c["gelu"])
    elif c["kind"] == "norm":
        H.hsa_qk_norm_rope(st["q"], st["k"], c["heads"], c["kv_heads"], c["head_dim"], st["q_out"], st["k_out"],
                           q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, rope=st["rope"], pos=st["pos"],
                           interleaved=c["interleaved"])
    elif c["kind"] == "plan":
        H.hsa_page_plan(st["past"], st["fresh"], c["page"], st["page_table"], st["free"], st["free_at"], st["cu"],
                        st["kv_lens"], st["pos"], st["slots"], st["free_next"])
    elif c["kind"] == "swap":
        H.hsa_cache_store(st["k"], st["v"], st["idx"], c["rows"], c["kv_heads"], st["k_cache"], st["v_cache"], st["k_exp"],
                          st["v_exp"])
        H.hsa_cache_load(st["k_cache"], st["v_cache"], st["idx"], c["rows"], c["kv_heads"], st["k_back"], st["v_back"],
                         st["k_exp"], st["v_exp"])
    else:
        dh = c["head_dim"]
        H.hsa_paged_attention(st["q"], st["k_cache"], st["v_cache"], st["page_table"], st["kv_lens"], c["page"],
                              c["heads"], c["kv_heads"], dh, dh ** -0.5, st["o"], st["workspace"], k_exp=st["k_exp"],
                              v_exp=st["v_exp"], lse=st["lse"])


def _rotated(y, rope, pos, interleaved):
    """The first channels of every head of y [n, heads, dh] turned by the rows `pos` of rope [positions, pairs, 2]."""
    pairs = rope.shape[1]
    cos, sin = rope[pos.long()][:, None].unbind(-1)  # [n, 1, pairs]
    x, rest = y[..., :2 * pairs], y[..., 2 * pairs:]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :pairs], x[..., pairs:])
    u, v = a * cos - b * sin, a * sin + b * cos
    x = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([x, rest], -1)


def _plain(st):
    c = st["case"]
    if c["kind"] == "linear":
        y = torch.matmul(st["x"].float(), _values(st["w"], st["w_exp"]).t())
        if st["scale"] is not None:
            y = y * st["scale"][:, None]
        if c["gelu"]:
            y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
        if st["residual"] is not None:
            y = y + st["residual"].float()
        st["y"].copy_(y)
        return
    if c["kind"] == "norm":
        for x, heads in (("q", c["heads"]), ("k", c["kv_heads"])):
            y = st[x].float().view(c["rows"], heads, -1)
            y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * st[x + "_weight"].float()
            if st["rope"] is not None:
                y = _rotated(y, st["rope"], st["pos"], c["interleaved"])
            st[x + "_out"].copy_(y.view(c["rows"], -1))
        return
    if c["kind"] == "plan":
        page, table, free = c["page"], st["page_table"], st["free"]
        past, fresh = st["past"].long(), st["fresh"].long()
        end = past + fresh
        have = (past + page - 1) // page
        need = (end + page - 1) // page - have
        cu, nu = torch.cumsum(fresh, 0), torch.cumsum(need, 0)
        first, count = st["free_at"][0].long(), st["free_at"][1].long()
        rank = torch.arange(table.shape[1], device=DEV)
        new = (rank >= have[:, None]) & (rank < (have + need)[:, None])
        at = (nu - need)[:, None] + rank - have[:, None]
        table.copy_(torch.where(new, torch.where(at < count, free[(first + at.clamp(min=0)) % free.numel()], -1), table))
        st["cu"].copy_(torch.cat([torch.zeros_like(cu[:1]), cu]))
        st["kv_lens"].copy_(end)
        t = torch.arange(st["tokens"], device=DEV)
        s = torch.searchsorted(cu, t, right=True)
        there = s < cu.numel()
        s = s.clamp(max=cu.numel() - 1)
        pos = past[s] + t - (cu - fresh)[s]
        pages = table[s, (pos // page).clamp(max=table.shape[1] - 1)].long()
        st["pos"].copy_(torch.where(there, pos, -1))
        st["slots"].copy_(torch.where(there & (pages >= 0), pages * page + pos % page, -1))
        taken = torch.minimum(nu[-1], count)
        st["free_next"].copy_(torch.stack([(first + taken) % free.numel(), count - taken, nu[-1] - taken]))
        return
    if c["kind"] == "swap":
        idx = st["idx"].long()
        for x in ("k", "v"):
            st[x + "_cache"][idx], st[x + "_exp"][idx] = _quantize(st[x])
            st[x + "_back"].copy_(_values(st[x + "_cache"][idx], st[x + "_exp"][idx]))
        return
    kv, dh, heads = c["kv_heads"], c["head_dim"], c["heads"]
    n, length, page = c["seqs"], st["page_table"].shape[1] * c["page"], c["page"]
    t = torch.arange(length, device=DEV)
    rows = (st["page_table"].long()[:, t // page] * page + t % page).view(-1)
    k, v = (_values(st[x + "_cache"][rows], st[x + "_exp"][rows]).view(n, length, kv, dh).transpose(1, 2) for x in ("k", "v"))
    s = torch.matmul(st["q"].float().view(n, kv, heads // kv, dh), k.transpose(-1, -2).contiguous()) * dh ** -0.5
    s.masked_fill_((t >= st["kv_lens"][:, None])[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = (s - m).exp()
    total = p.sum(-1, keepdim=True)
    st["o"].copy_((torch.matmul(p, v) / total).reshape(n, heads * dh))
    st["lse"].copy_((m + total.log()).reshape(n, heads))


OUTPUTS = {"linear": ("y",), "norm": ("q_out", "k_out"), "plan": ("page_table", "cu", "kv_lens", "pos", "slots", "free_next"),
           "swap": ("k_back", "v_back", "k_exp", "v_exp"), "paged": ("o", "lse")}


def run(st):
    if own:
        _own(st)
    else:
        _plain(st)
    return [st[x] for x in OUTPUTS[st["case"]["kind"]]]


def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "linear":
        rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
        out = (2 if case["out"] == "bf16" else 4) * rows * d_out
        return {"bytes": d_out * d_in // 2 + d_out * d_in // GROUP + rows * d_in * es + out * (2 if case["residual"] else 1) +
                (4 * rows if case["scaled"] else 0), "flops": 2 * rows * d_in * d_out}
    if case["kind"] == "plan":
        past, fresh = _plan_lengths(case)
        page = case["page"]
        new = sum(-(-(p + f) // page) - -(-p // page) for p, f in zip(past, fresh))
        # lengths in, offsets and lengths out; a position and a row for each token; new pages from the ring into the table,
        # and the old last page of sequences that go on in it
        old = sum(1 for p, f in zip(past, fresh) if p % page and f)
        return {"bytes": 16 * len(past) + 8 * (sum(fresh) + case["pad"]) + 8 * new + 4 * old + 28, "flops": 0}
    kv, dh = case["kv_heads"], case["head_dim"]
    row = kv * dh
    held = row // 2 + row // GROUP
    if case["kind"] == "norm":
        n, rot = case["rows"], case["rope_dim"]
        return {"bytes": 2 * n * (case["heads"] * dh + row) * es + 4 * n + 2 * dh * es + min(n, case["positions"]) * rot * 4,
                "flops": 0}
    if case["kind"] == "swap":
        return {"bytes": 2 * case["rows"] * (2 * (row * es + held) + 4), "flops": 0}
    lens, d = spread(case["seqs"], case["shortest"], case["longest"]), case["heads"] * dh
    return {"bytes": 2 * sum(lens) * held + len(lens) * (2 * d * es + 4 * case["heads"] + 4) +
            4 * sum(-(-x // case["page"]) for x in lens), "flops": 4 * sum(lens) * d}


def _codes64(codes, ex):
    """Values of rows of codes by their fields: a sign, 2 exponent bits of bias 1, 1 fraction bit; times 2^ex."""
    b = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    e, f = (b >> 1) & 3, (b & 1).double()
    mag = torch.where(e == 0, f / 2, (1 + f / 2) * torch.pow(2.0, (e - 1).double()))
    y = torch.where(b >= 8, -mag, mag).view(*ex.shape, GROUP)
    return (y * torch.pow(2.0, ex.double())[..., None]).flatten(-2)


def _nearest64(x):
    """The nearest of a group's values to each of x, and the exponents: by the distances to all, ties to the even code."""
    y = x.double().view(*x.shape[:-1], -1, GROUP)
    top = y.abs().amax(-1)
    ex = torch.ceil(torch.log2(top / 6)).clamp(EXP_MIN, EXP_MAX)
    ex = torch.where((6 * torch.pow(2.0, ex) < top) & (ex < EXP_MAX), ex + 1, ex)
    ex = torch.where((6 * torch.pow(2.0, ex - 1) >= top) & (ex > EXP_MIN), ex - 1, ex)
    y = y * torch.pow(2.0, -ex)[..., None]
    best, off = torch.zeros_like(y), torch.full_like(y, math.inf)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):  # even codes first: of two equally near ones the even one stays
        value = (0, .5, 1, 1.5, 2, 3, 4, 6)[i]
        d = (y.abs() - value).abs()
        best, off = torch.where(d < off, value, best), torch.minimum(d, off)
    best = torch.where(y < 0, -best, best)
    return (best * torch.pow(2.0, ex)[..., None]).flatten(-2), ex


def exact(case, seed):
    """The outputs from the definitions, in 64 bits."""
    st = prepare(case, seed)
    if case["kind"] == "linear":
        x, turn = st["x"].double(), max(1, (1 << 25) // case["d_in"])
        y = torch.cat([x @ _codes64(st["w"][a:a + turn], st["w_exp"][a:a + turn]).t().contiguous()
                       for a in range(0, case["d_out"], turn)], 1)
        if case["scaled"]:
            y = y * st["scale"].double()[:, None]
        if case["gelu"]:
            y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
        if case["residual"]:
            y = y + st["residual"].double()
        return [y]
    if case["kind"] == "norm":
        out = []
        for x, heads in (("q", case["heads"]), ("k", case["kv_heads"])):
            y = st[x].double().reshape(case["rows"], heads, -1)
            y = y * (y.square().sum(-1, keepdim=True) / y.shape[-1] + EPS).rsqrt() * st[x + "_weight"].double()
            rot = case["rope_dim"]
            if rot:
                i = torch.arange(rot // 2, device=DEV)
                one, two = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
                z = torch.complex(y[..., one], y[..., two]) * torch.view_as_complex(st["rope"].double()[st["pos"].long()])[:, None]
                y[..., one], y[..., two] = z.real, z.imag
            out.append(y.view(case["rows"], -1))
        return out
    if case["kind"] == "plan":
        past, fresh = _plan_lengths(case)
        page, table, free = case["page"], st["page_table"].cpu(), st["free"].tolist()
        at, left, _ = st["free_at"].tolist()
        cu, pos, slots = [0], [], []
        for s, (p, f) in enumerate(zip(past, fresh)):
            row = table[s].tolist()
            for j in range(-(-p // page), -(-(p + f) // page)):
                row[j], at, left = free[at], (at + 1) % len(free), left - 1
            table[s] = torch.tensor(row, dtype=torch.int32)
            cu.append(cu[-1] + f)
            pos += range(p, p + f)
            slots += [row[i // page] * page + i % page for i in range(p, p + f)]
        pos, slots = (x + [-1] * case["pad"] for x in (pos, slots))
        return [table] + [torch.tensor(x, dtype=torch.int32)
                          for x in (cu, [p + f for p, f in zip(past, fresh)], pos, slots, [at, left, 0])]
    if case["kind"] == "swap":
        (k, ke), (v, ve) = _nearest64(st["k"]), _nearest64(st["v"])
        return [k, v, None, None]
    kv, dh, heads, page = case["kv_heads"], case["head_dim"], case["heads"], case["page"]
    os, ls = [], []
    for i, m in enumerate(spread(case["seqs"], case["shortest"], case["longest"])):
        t = torch.arange(m, device=DEV)
        rows = st["page_table"][i].long()[t // page] * page + t % page
        q = st["q"][i].double().view(kv, heads // kv, dh)
        k, v = (_codes64(st[x + "_cache"][rows], st[x + "_exp"][rows]).view(m, kv, dh).transpose(0, 1).contiguous() for x in ("k", "v"))
        s = (q[:, :, None] * k[:, None]).sum(-1) * dh ** -0.5 if m < 64 else \
            torch.stack([q[h] @ k[h].t().contiguous() for h in range(kv)]) * dh ** -0.5
        lse = torch.logsumexp(s, -1)
        o = torch.stack([torch.exp(s[h] - lse[h, :, None]) @ v[h] for h in range(kv)])
        os.append(o.view(1, heads * dh))
        ls.append(lse.view(1, heads))
    return [torch.cat(os), torch.cat(ls)]
