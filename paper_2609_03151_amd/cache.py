"""The key-value cache of one rank's heads, in pages.

A rank of a BASP group holds K and V of the whole sequence for its H_kv/G heads after the head
exchange (Sec. II-C of the paper).  `PagedKV` keeps them for generation: every new token's K and V
are written behind the others' and its query attends to all of them, on the rank's heads, with no
exchange of cached tokens.  A sequence's tokens lie in pages of `page` tokens, listed in its row
of a block table; which page a sequence gets is the caller's.

In 8 bits (`torch.float8_e4m3fn`) a token of one head is stored as e4m3 values with one
power-of-two scale 2^e, at half the bytes (129 for 256 at d = 128).  A value is off by at most 2^-4 of
itself, or by 2^-10 * 2^e if that is more: values below 2^-6 * 2^e keep fewer bits, and those below
2^-10 * 2^e are stored as 0.  The row's largest is above 224 * 2^e (or e is -110, its least).
"""
from __future__ import annotations

import torch

from . import attn_decode, attn_decode_shared, kv_read, kv_write


class PagedKV:
    def __init__(self, n_pages: int, n_kv: int, d: int, page: int = 64,
                 dtype: torch.dtype = torch.bfloat16, device="cuda"):
        self.page = page
        shape = (n_pages, n_kv, page, d)
        # contents are read only where a write has been
        self.k_pages = torch.empty(shape, dtype=dtype, device=device)
        self.v_pages = torch.empty(shape, dtype=dtype, device=device)
        self.k_scales = self.v_scales = None
        if dtype == torch.float8_e4m3fn:
            self.k_scales = torch.empty(shape[:3], dtype=torch.uint8, device=device)
            self.v_scales = torch.empty(shape[:3], dtype=torch.uint8, device=device)

    def write(self, k, v, block_table, start, count=None):
        """K, V [b, T, n_kv, d] of T new tokens per sequence at positions start[s] .. (`kv_write`)."""
        kv_write(k, v, self.k_pages, self.v_pages, block_table, start, count=count,
                 k_scales=self.k_scales, v_scales=self.v_scales)

    def read(self, block_table, T: int, start=None, count=None):
        """(K, V) [b, T, n_kv, d] of positions start[s] .. start[s] + count[s] - 1 (`kv_read`)."""
        return kv_read(self.k_pages, self.v_pages, block_table, T, start=start, count=count,
                       k_scales=self.k_scales, v_scales=self.v_scales)

    def attend(self, q, block_table, lens, scale: float | None = None, max_len: int | None = None,
               out=None, lse=None, workspace=None):
        """(O [b, n_q, d], LSE [b, n_q]) of one new token per sequence over its first lens[s] tokens
        (`attn_decode`)."""
        return attn_decode(q, self.k_pages, self.v_pages, block_table, lens, scale=scale,
                           max_len=max_len, k_scales=self.k_scales, v_scales=self.v_scales,
                           out=out, lse=lse, workspace=workspace)

    def attend_shared(self, q, block_table, lens, groups=None, prefix_lens=None,
                      scale: float | None = None, max_len: int | None = None,
                      cap: float | None = None, slopes=None, out=None, lse=None, workspace=None):
        """The same for sequences in groups that share a prefix, and with scores capped and biased by
        distance (`attn_decode_shared`)."""
        return attn_decode_shared(q, self.k_pages, self.v_pages, block_table, lens, groups,
                                  prefix_lens, scale=scale, max_len=max_len, cap=cap,
                                  slopes=slopes, k_scales=self.k_scales, v_scales=self.v_scales,
                                  out=out, lse=lse, workspace=workspace)
