"""Attention over a quantized cache, as a decoder runs it with whole prompts and
drafted tokens.

Whole prompts come packed, back to back: soniq_kv_plan has said where their
tokens go, they attend to themselves in 16 bits (soniq_prompt_attend), and their
keys and values are put into the cache.  A later step takes the hidden states of
T tokens of each sequence: a piece of a prompt, one new token, or a tree of
drafted ones.  The fused projection runs on the library's quantized matmul (signed
activations, Eq. (1), one scale per token), queries and keys are normalised and
turned by their positions where the layer does so (soniq_rotate_heads), keys and
values go to the cache (soniq_kv_write), the queries attend over the cached
context and over the drafts their mask shows (soniq_kv_attend), and the output
projection closes the layer.  When the drafts have been judged, `accept` moves the
rows of the accepted path behind the context; they are quantized from the same
16-bit rows again, so a token's codes do not depend on whether it was drafted.

This module sequences the calls and does the integer bookkeeping of drafts; every
arithmetic step runs in the library's kernels.  The layer is fp16; a model that
runs in bf16 makes the same calls itself."""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import soniq as sq


class CachedAttention:
    """One attention layer and its cache.

    qkv, out: dicts with W (fp32 [N][K], numpy or torch), perm, count, bits (as
    the workloads module makes them).  qkv's rows are the query heads (q_heads
    of k.D), the key heads and the value heads; out's channels the query heads
    (of v.D).  The cache has n_pages pages of page_size tokens.  rotary, gains,
    eps: sq.rotate_heads' of the queries and keys (gains: a pair, fp32 [k.D] each),
    left out: queries and keys stay as projected."""

    def __init__(self, qkv: dict, out: dict, q_heads: int, k: sq.KVLayout, v: sq.KVLayout, n_pages: int,
                 page_size: int = 64, device="cuda", rotary: Optional[sq.Rotary] = None,
                 gains: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, eps: float = 1e-6):
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
        self.q = self.k = self.v = self.o = self.at = None
        self.rotary, self.gains, self.eps = rotary, gains or (None, None), eps

    def _project(self, which: int, x: torch.Tensor) -> torch.Tensor:
        layout, Wp, s_w = self.weights[which]
        Ap, s_a = sq.quantize_act(layout, x, "row")
        return sq.mp_gemm(layout, Ap, s_a, Wp, s_w, scale_mode="row")

    def _heads(self, X: torch.Tensor, positions):
        """Queries, keys and values [n][heads][..] of the rows X [n][K]; positions: a
        function that gives the rows' (called where they are used)."""
        q, k, v = self._project(0, X).split(self.widths, dim=-1)
        q = q.unflatten(-1, (self.q_heads, self.cache.k.D))
        k = k.unflatten(-1, (self.cache.heads, self.cache.k.D))
        if self.rotary is not None or self.gains[0] is not None or self.gains[1] is not None:
            sq.rotate_heads(self.rotary, q, k, positions() if self.rotary is not None else None, *self.gains, self.eps,
                            q_out=q, k_out=k)
        return q, k, v.unflatten(-1, (self.cache.heads, self.cache.v.D))

    def prompt(self, X: torch.Tensor, step: sq.KVStep) -> torch.Tensor:
        """Whole prompts, packed.  X: fp16 [n][K], as many rows as the step's buffers
        (sq.kv_plan from lengths of 0 or less; sequences that add nothing may stand
        among them); rows behind the step's tokens are padding.  Returns fp16 [n][N]."""
        self.q, self.k, self.v = self._heads(X, lambda: step.positions)
        sq.kv_write(self.cache, self.k, self.v, step.slots)
        self.o = torch.zeros(X.shape[0], self.q_heads, self.cache.v.D, dtype=X.dtype, device=X.device)
        sq.prompt_attend(self.q, self.k, self.v, step.starts, out=self.o)
        return self._project(1, self.o.view(X.shape[0], -1))

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

    def planned(self, plan: sq.KVStep, B: int, T: int) -> torch.Tensor:
        """The slots of a plan's tokens, which stand packed, as int64 [B][T]: row b those of
        its sequence b; -1 in sequences that add none or were not served.  One that adds
        another number than T has no place in such a step: its slots are beyond the cache,
        which the library reports."""
        if plan.starts.numel() <= B:
            raise ValueError("the plan has fewer sequences than the step")
        none = self.cache.n_pages * self.cache.page_size
        n = plan.slots.numel()
        if n == 0:
            return torch.full((B, T), -1, dtype=torch.int64, device=plan.slots.device)
        first, count = plan.starts[:B, None].long(), (plan.starts[1:B + 1] - plan.starts[:B])[:, None]
        slots = plan.slots[(first + torch.arange(T, device=first.device)).clamp(max=n - 1)]
        served = (count > 0) & (plan.slots[first.clamp(max=n - 1)] >= 0)
        return torch.where(served, torch.where(count == T, slots, none), -1)

    def step(self, X: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
             mask: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
             slots: Union[None, torch.Tensor, sq.KVStep] = None) -> torch.Tensor:
        """X: fp16 [B][T][K]; page_table int32 [B][pages]; lengths int32 [B] (the
        context in front of the T tokens); mask as sq.kv_attend's.  positions: int32
        [B][T], what a layer with a rotary turns by (left out: one after the other
        behind the context; of a tree's drafts those with the same depth share one).
        slots: where the tokens go: sq.kv_plan's step, each of whose first B sequences adds
        T tokens or none; or int64 [B][T] (not a plan's own packed list, in which absent
        sequences have no place).  A sequence none of whose slots is in the cache is absent
        from the step.  Left out, the table says where: not behind sq.kv_plan, which leaves pages
        that were given back in it, and sequences that wait without.  Returns fp16
        [B][T][N]; q, k, v and the attention's output stay in self."""
        B, T, K = X.shape
        if slots is None:
            at = self.slots(page_table, lengths, T)
        elif isinstance(slots, sq.KVStep):
            at = self.planned(slots, B, T)
        elif slots.numel() == B * T:
            at = slots.reshape(B, T)
        else:
            raise ValueError("slots must be a KVStep or int64 [B][T]")
        seen = lengths
        if slots is not None:
            there = ((at >= 0) & (at < self.cache.n_pages * self.cache.page_size)).any(1)
            lengths = torch.where(there, lengths.clamp(min=0), lengths)       # (one that begins may have a negative length)
            seen = torch.where(there, lengths, -1)

        def where():
            p = lengths[:, None] + torch.arange(T, dtype=torch.int32, device=X.device) if positions is None else positions
            return p.to(torch.int32).reshape(-1)

        q, k, v = self._heads(X.reshape(B * T, K), where)
        self.q, self.k, self.v = (t.unflatten(0, (B, T)) for t in (q, k, v))
        self.at = at
        sq.kv_write(self.cache, k, v, at.view(-1))
        self.o = sq.kv_attend(self.cache, self.q, page_table, seen, mask)
        return self._project(1, self.o.view(B * T, -1)).view(B, T, -1)

    def accept(self, path: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
        """path: int64 [B][A], the accepted drafts of the last step in their order,
        -1 behind the last.  Their rows become the context's next tokens; returns
        the new lengths.  Nothing is written but slots of that step: a sequence that was
        absent from it (the page behind its context may be another's) keeps its length."""
        B, T = self.k.shape[:2]
        lengths = torch.where((self.at >= 0).any(1), lengths.clamp(min=0), lengths)
        slots = self.slots(page_table, lengths, path.shape[1])
        slots = torch.where((slots[:, :, None] == self.at[:, None]).any(2), slots, -1)
        to = torch.full((B, T + 1), -1, dtype=torch.int64, device=path.device)
        to.scatter_(1, torch.where(path >= 0, path, T), slots)
        sq.kv_write(self.cache, self.k.flatten(0, 1), self.v.flatten(0, 1), to[:, :T].reshape(-1).contiguous())
        return (lengths + ((path >= 0) & (slots >= 0)).sum(1)).to(torch.int32)

    def context(self, page_table: torch.Tensor, lengths: torch.Tensor, b: int) -> Tuple[torch.Tensor, torch.Tensor]:
        """The keys [n][heads][D] and values that the cache holds of sequence b."""
        n = max(int(lengths[b]), 0)
        zero = torch.zeros(1, dtype=torch.int32, device=lengths.device)
        return sq.kv_read(self.cache, self.slots(page_table[b:b + 1], zero, n).view(-1))
