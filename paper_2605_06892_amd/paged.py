"""A paged key/value cache of one attention layer and the two steps over it.

Strings the calls over several sequences together in stream order:

    prefill   hsa_packed_attention   the prompts attend to themselves, causally
              hsa_cache_store        their keys and values go to their pages
    decode    hsa_cache_store        every sequence's new row goes to its page
              hsa_paged_attention    one new token per sequence attends to its pages

The cache has n_pages * page_size rows, kept in their own type or in 8 bits; which
page belongs to which sequence is the caller's: a table of page numbers per
sequence, on the host for `slots` and on the device for `decode`. Buffers are
allocated once with torch and owned by the caller; nothing here computes.
"""

from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

from . import hsa_step as H


@dataclass
class PagedCache:
    k: torch.Tensor            # [n_pages * page_size, kv_heads * head_dim]: the dtype, or float8_e4m3fn codes
    v: torch.Tensor
    k_exp: torch.Tensor | None  # int8 [n_pages * page_size, kv_heads] with codes
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
                 device="cuda", e4m3: bool = False, workspace: torch.Tensor | None = None) -> "PagedCache":
        """e4m3 keeps the rows in 8 bits (one exponent per row and head), half of bf16's bytes. workspace: another
        layer's cache's, for layers whose steps follow each other in one stream; None allocates one."""
        rows, d = n_pages * page_size, kv_heads * head_dim
        e = lambda *s, dt=dtype: torch.empty(*s, dtype=dt, device=device)  # noqa: E731
        held = torch.float8_e4m3fn if e4m3 else dtype
        exps = [e(rows, kv_heads, dt=torch.int8) if e4m3 else None for _ in range(2)]
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
