"""A paged key/value cache of one attention layer and the two steps over it.

Strings the calls over several sequences together in stream order:

    prefill   hsa_packed_attention   the prompts attend to themselves, causally
              hsa_cache_store        their keys and values go to their pages
    decode    hsa_cache_store        every sequence's new row goes to its page
              hsa_paged_attention    one new token per sequence attends to its pages

The cache has n_pages * page_size rows, kept in their own type or in 8 or 4 bits; which
page belongs to which sequence is the caller's: a table of page numbers per
sequence, on the host for `slots` and on the device for `decode`, or a `PagePool`,
which hands pages out on the device:

    plan      hsa_page_plan          pages, cache rows and positions of every sequence's fresh tokens

`Layer4` is a whole attention layer of such a program, its weights in 4 bits:

    project   hsa_row_rms_scale, hsa_linear_w4   queries, keys and values of the normed rows
              hsa_qk_norm_rope                   their heads normed and rotated, where they lie
    attend    prefill or decode
    project   hsa_linear_w4                      back, and the residual

Buffers are allocated once with torch and owned by the caller; nothing here computes, but for a count of lacking pages.
"""

from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

from . import hsa_step as H


@dataclass
class PagedCache:
    k: torch.Tensor            # [n_pages * page_size, kv_heads * head_dim]: the dtype, or float8_e4m3fn codes;
    v: torch.Tensor            # e2m1 codes: uint8, half as wide
    k_exp: torch.Tensor | None  # int8 [n_pages * page_size, kv_heads] with codes, kv_heads * head_dim / 32 with e2m1
    v_exp: torch.Tensor | None
    workspace: torch.Tensor    # uint8, the decoding step's; steps that may overlap in time need one each
    page_size: int
    kv_heads: int
    head_dim: int

    @property
    def n_pages(self) -> int:
        return self.k.shape[0] // self.page_size

    @property
    def scale(self) -> float:
        return self.head_dim ** -0.5

    @classmethod
    def allocate(cls, n_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype: torch.dtype,
                 device="cuda", e4m3: bool = False, workspace: torch.Tensor | None = None,
                 e2m1: bool = False) -> "PagedCache":
        """e4m3 keeps the rows in 8 bits (one exponent per row and head), half of bf16's bytes, e2m1 in 4 (one exponent
        per 32 values), 17/64 of them. workspace: another layer's cache's, for layers whose steps follow each other in
        one stream; None allocates one."""
        if e4m3 and e2m1:
            raise ValueError("rows are kept in 8 bits or in 4")
        rows, d = n_pages * page_size, kv_heads * head_dim
        e = lambda *s, dt=dtype: torch.empty(*s, dtype=dt, device=device)  # noqa: E731
        held = torch.float8_e4m3fn if e4m3 else torch.uint8 if e2m1 else dtype
        exps = [e(rows, d // 32 if e2m1 else kv_heads, dt=torch.int8) if e4m3 or e2m1 else None for _ in range(2)]
        d = d // 2 if e2m1 else d
        if workspace is None:
            workspace = e(H.PAGED_WORKSPACE_BYTES, dt=torch.uint8)
        return cls(k=e(rows, d, dt=held), v=e(rows, d, dt=held), k_exp=exps[0], v_exp=exps[1], workspace=workspace,
                   page_size=page_size, kv_heads=kv_heads, head_dim=head_dim)


def slots(page_table: np.ndarray, page_size: int, seqs, positions) -> np.ndarray:
    """Cache rows (int32) of the tokens at `positions` of sequences `seqs`, by the host's table of pages. -1 (no row)
    for a negative sequence, position or page number, and for a page whose rows do not fit int32."""
    seqs, positions = np.asarray(seqs), np.asarray(positions)
    pages = page_table[np.maximum(seqs, 0), np.maximum(positions, 0) // page_size].astype(np.int64)
    rows = pages * page_size + positions % page_size
    return np.where((seqs < 0) | (positions < 0) | (pages < 0) | (rows > 2 ** 31 - 1), -1, rows).astype(np.int32)


def prefill(c: PagedCache, q, k, v, cu, idx, heads: int, o, lse=None) -> None:
    """Whole prompts, packed: o = causal attention within cu[s] .. cu[s+1], and row idx[j] of the cache = row j of
    k and v (the slots of their tokens)."""
    H.hsa_packed_attention(q, k, v, cu, cu, heads, c.kv_heads, c.head_dim, c.scale, True, o, lse=lse)
    H.hsa_cache_store(k, v, idx, k.shape[0], c.kv_heads, c.k, c.v, c.k_exp, c.v_exp)


def decode(c: PagedCache, q, k, v, idx, page_table, kv_lens, heads: int, o, lse=None) -> None:
    """One new token per sequence: its keys and values to row idx[s] (-1: none), then its attention to the
    kv_lens[s] rows of its pages, the new one among them."""
    H.hsa_cache_store(k, v, idx, k.shape[0], c.kv_heads, c.k, c.v, c.k_exp, c.v_exp)
    H.hsa_paged_attention(q, c.k, c.v, page_table, kv_lens, c.page_size, heads, c.kv_heads, c.head_dim, c.scale, o,
                          c.workspace, k_exp=c.k_exp, v_exp=c.v_exp, lse=lse)


@dataclass
class PagePool:
    """The pages of many sequences, handed out on the device: all int32, and changed in place by `plan`."""

    page_table: torch.Tensor  # [n_seqs, max_pages]
    lens: torch.Tensor        # [n_seqs]: rows that each sequence has
    free: torch.Tensor        # [n_pages]: a ring of the free pages
    free_at: torch.Tensor     # [3]: its first free entry, how many there are, and how many pages were lacking
    cu: torch.Tensor          # [n_seqs + 1]: the fresh tokens' offsets,
    pos: torch.Tensor         # [n_tokens]: their positions
    slots: torch.Tensor       # [n_tokens]: and their cache rows; -1 behind the last
    page_size: int
    lacked: torch.Tensor | None = None  # [1]: pages that were lacking in all steps since the caller last set it to 0

    def __post_init__(self):
        if self.lacked is None:
            self.lacked = torch.zeros(1, dtype=torch.int32, device=self.free_at.device)

    @classmethod
    def allocate(cls, n_pages: int, page_size: int, n_seqs: int, max_pages: int, n_tokens: int, device="cuda") -> "PagePool":
        """n_tokens: the most fresh tokens of one step."""
        i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)  # noqa: E731
        return cls(page_table=i(n_seqs, max_pages) - 1, lens=i(n_seqs),
                   free=torch.arange(n_pages, dtype=torch.int32, device=device),
                   free_at=torch.tensor([0, n_pages, 0], dtype=torch.int32, device=device), cu=i(n_seqs + 1),
                   pos=i(n_tokens), slots=i(n_tokens), page_size=page_size)

    def plan(self, fresh: torch.Tensor) -> None:
        """fresh[s] more tokens for every sequence: their pages, positions and rows, and the new lengths. A step that finds too
        few pages says so in free_at[2], and `lacked` keeps count of them over the steps. A page that was lacking is not
        asked for again: the tokens in it, the later steps' too, have slot -1 and are left out by attention, until `resume`."""
        H.hsa_page_plan(self.lens, fresh, self.page_size, self.page_table, self.free, self.free_at, self.cu, self.lens,
                        self.pos, self.slots, self.free_at)
        self.lacked.add_(self.free_at[2:])

    def release(self, seq: int) -> None:
        """A finished sequence's pages go back to the ring, and its length to 0. Waits for the device."""
        self._cut(seq, 0)

    def resume(self, seq: int) -> int:
        """A sequence that was lacking a page goes back to the rows before it: what pages it has behind them go back to the
        ring. Returns how many of its last tokens are to be planned and computed again; 0 if it has all its pages. Waits
        for the device."""
        rows = int(self.lens[seq])
        gone = (self.page_table[seq, :-(-rows // self.page_size)] < 0).nonzero()
        if len(gone) == 0:
            return 0
        keep = int(gone[0]) * self.page_size
        self._cut(seq, keep)
        return rows - keep

    def _cut(self, seq: int, rows: int) -> None:
        """Length `rows`, a multiple of the page size, and what pages are behind it to the ring."""
        first, n = rows // self.page_size, -(-int(self.lens[seq]) // self.page_size)
        pages = self.page_table[seq, first:n]
        pages = pages[pages >= 0]
        at = int(self.free_at[0]) + int(self.free_at[1])
        self.free[(torch.arange(len(pages), device=pages.device) + at) % len(self.free)] = pages
        self.free_at[1] += len(pages)
        self.page_table[seq, first:n] = -1
        self.lens[seq] = rows


@dataclass
class Layer4:
    """An attention layer with weights in 4 bits: x + out(attention(norm_rope(qkv(rms(x)))))."""

    w_qkv: tuple             # codes and exponents (hsa_quantize_w4) of [(heads + 2 kv_heads) * head_dim, d]
    w_out: tuple             # of [d, heads * head_dim]
    q_norm: torch.Tensor | None  # [head_dim]
    k_norm: torch.Tensor | None
    heads: int
    kv_heads: int
    head_dim: int
    scale: torch.Tensor      # fp32 [n_tokens]
    qkv: torch.Tensor        # [n_tokens, (heads + 2 kv_heads) * head_dim]
    o: torch.Tensor          # [n_tokens, heads * head_dim]

    @classmethod
    def allocate(cls, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, head_dim: int, n_tokens: int,
                 q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None) -> "Layer4":
        """From weights of the model's dtype, for steps of at most n_tokens tokens."""
        def held(w):
            codes = torch.empty(w.shape[0], w.shape[1] // 2, dtype=torch.uint8, device=w.device)
            exps = torch.empty(w.shape[0], w.shape[1] // 32, dtype=torch.int8, device=w.device)
            H.hsa_quantize_w4(w, codes, exps)
            return codes, exps

        e = lambda *s, dt=w_qkv.dtype: torch.empty(*s, dtype=dt, device=w_qkv.device)  # noqa: E731
        return cls(w_qkv=held(w_qkv), w_out=held(w_out), q_norm=q_norm, k_norm=k_norm, heads=heads, kv_heads=kv_heads,
                   head_dim=head_dim, scale=e(n_tokens, dt=torch.float32), qkv=e(n_tokens, w_qkv.shape[0]),
                   o=e(n_tokens, heads * head_dim))

    def step(self, x: torch.Tensor, c: PagedCache, pool: PagePool, rope: torch.Tensor | None, y: torch.Tensor,
             prompts: bool = False) -> None:
        """y = the layer's output for the tokens x of pool.plan's last step: exactly one for every sequence, in their
        order (fresh was 1 throughout; an ended sequence goes on with any token and is released when another
        takes its place), or with `prompts` any number, where sequences begin (they attend to themselves
        only). Rows of a page that was lacking are left out, the newest among them (`PagePool.resume`). y may be x.
        ValueError, with nothing enqueued, for more tokens than the layer or the pool was made for, a decoding step of
        another number of tokens, and a y of other sizes than x."""
        n = x.shape[0]
        if n > min(len(self.scale), len(self.qkv), len(self.o), len(pool.pos)):
            raise ValueError(f"the layer takes {len(self.scale)} tokens a step and the pool plans {len(pool.pos)}, got {n}")
        if not prompts and n != len(pool.lens):
            raise ValueError(f"a decoding step has one token for each of {len(pool.lens)} sequences, got {n}")
        if y.shape != x.shape:
            raise ValueError("y is as large as x")
        q_width, kv_width = self.heads * self.head_dim, self.kv_heads * self.head_dim
        qkv, o = self.qkv[:n], self.o[:n]
        H.hsa_row_rms_scale(x, n, self.scale)
        H.hsa_linear_w4(x, n, *self.w_qkv, qkv, row_scale=self.scale)
        q, k, v = qkv.split([q_width, kv_width, kv_width], dim=1)
        H.hsa_qk_norm_rope(q, k, self.heads, self.kv_heads, self.head_dim, q, k, self.q_norm, self.k_norm, rope=rope,
                           pos=pool.pos[:n])
        if prompts:
            prefill(c, q, k, v, pool.cu, pool.slots, self.heads, o)
        else:
            decode(c, q, k, v, pool.slots, pool.page_table, pool.lens, self.heads, o)
        H.hsa_linear_w4(o, n, *self.w_out, y, residual=x)
