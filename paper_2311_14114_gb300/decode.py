"""Attention over a quantized cache, as a decoder runs it with drafted tokens.

A step takes the hidden states of T tokens of each sequence: a piece of a
prompt, one new token, or a tree of drafted ones.  The fused projection runs on
the library's quantized matmul (signed activations, Eq. (1), one scale per
token), its keys and values go to the cache (soniq_kv_write), the queries
attend over the cached context and over the drafts their mask shows
(soniq_kv_attend), and the output projection closes the layer.  When the
drafts have been judged, `accept` moves the rows of the accepted path behind
the context; they are quantized from the same 16-bit rows again, so a token's
codes do not depend on whether it was drafted.

This module sequences the calls and does the integer bookkeeping of slots;
every arithmetic step runs in the library's kernels.  The layer is fp16 and
applies no position encoding: there is no place for one between its projection
and its cache.  A model that turns q and k by their positions, or runs in bf16,
makes the same calls itself."""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import soniq as sq


class CachedAttention:
    """One attention layer and its cache.

    qkv, out: dicts with W (fp32 [N][K], numpy or torch), perm, count, bits (as
    the workloads module makes them).  qkv's rows are the query heads (q_heads
    of k.D), the key heads and the value heads; out's channels the query heads
    (of v.D).  The cache has n_pages pages of page_size tokens."""

    def __init__(self, qkv: dict, out: dict, q_heads: int, k: sq.KVLayout, v: sq.KVLayout, n_pages: int,
                 page_size: int = 64, device="cuda"):
        self.q_heads = int(q_heads)
        self.cache = sq.KVCache(k, v, n_pages, page_size, torch.float16, device=device)
        self.weights = []
        for lay in (qkv, out):
            layout = sq.Layout(lay["perm"], lay["count"], lay["bits"], act_kind=(sq.ACT_SIGNED, sq.ACT_SIGNED),
                               device=device)
            W = torch.as_tensor(lay["W"], dtype=torch.float32).to(device).contiguous()
            self.weights.append((layout,) + sq.pack_weights(layout, W))
        widths = (self.q_heads * k.D, k.heads * k.D, k.heads * v.D)
        if self.weights[0][1].shape[0] != sum(widths) or self.weights[1][0].K != self.q_heads * v.D:
            raise ValueError("the projections' sizes differ from the heads'")
        self.widths = widths
        self.q = self.k = self.v = self.o = None

    def _project(self, which: int, x: torch.Tensor) -> torch.Tensor:
        layout, Wp, s_w = self.weights[which]
        Ap, s_a = sq.quantize_act(layout, x, "row")
        return sq.mp_gemm(layout, Ap, s_a, Wp, s_w, scale_mode="row")

    def slots(self, page_table: torch.Tensor, lengths: torch.Tensor, T: int) -> torch.Tensor:
        """Slots (int64 [B][T]) of the T tokens behind each context; -1 in absent
        sequences; beyond the table, or where its page is none of the cache's, one that
        is no slot, which the library reports."""
        page = self.cache.page_size
        pos = lengths.long()[:, None] + torch.arange(T, device=lengths.device)
        entry = pos.clamp(min=0) // page
        inside = entry < page_table.shape[1]
        pages = page_table.long().gather(1, entry.clamp(max=page_table.shape[1] - 1))
        slot = torch.where(inside & (pages >= 0), pages * page + pos % page, self.cache.n_pages * page)
        return torch.where(lengths[:, None] >= 0, slot, -1)

    def step(self, X: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
             mask: Optional[torch.Tensor] = None) -> torch.Tensor:
        """X: fp16 [B][T][K]; page_table int32 [B][pages]; lengths int32 [B] (the
        context in front of the T tokens); mask as sq.kv_attend's.  Returns fp16
        [B][T][N]; q, k, v and the attention's output stay in self."""
        B, T, K = X.shape
        y = self._project(0, X.reshape(B * T, K)).view(B, T, -1)
        q, k, v = y.split(self.widths, dim=-1)
        self.q = q.unflatten(-1, (self.q_heads, self.cache.k.D))
        self.k = k.unflatten(-1, (self.cache.heads, self.cache.k.D))
        self.v = v.unflatten(-1, (self.cache.heads, self.cache.v.D))
        sq.kv_write(self.cache, self.k.flatten(0, 1), self.v.flatten(0, 1),
                    self.slots(page_table, lengths, T).view(-1))
        self.o = sq.kv_attend(self.cache, self.q, page_table, lengths, mask)
        return self._project(1, self.o.view(B * T, -1)).view(B, T, -1)

    def accept(self, path: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
        """path: int64 [B][A], the accepted drafts of the last step in their order,
        -1 behind the last.  Their rows become the context's next tokens; returns
        the new lengths."""
        B, T = self.k.shape[:2]
        to = torch.full((B, T + 1), -1, dtype=torch.int64, device=path.device)
        to.scatter_(1, torch.where(path >= 0, path, T), self.slots(page_table, lengths, path.shape[1]))
        sq.kv_write(self.cache, self.k.flatten(0, 1), self.v.flatten(0, 1), to[:, :T].reshape(-1))
        return torch.where(lengths >= 0, lengths + (path >= 0).sum(1), lengths).to(torch.int32)

    def context(self, page_table: torch.Tensor, lengths: torch.Tensor, b: int) -> Tuple[torch.Tensor, torch.Tensor]:
        """The keys [n][heads][D] and values that the cache holds of sequence b."""
        n = max(int(lengths[b]), 0)
        zero = torch.zeros(1, dtype=torch.int32, device=lengths.device)
        return sq.kv_read(self.cache, self.slots(page_table[b:b + 1], zero, n).view(-1))
