"""New requests beside running edit sessions: how their tokens get into the paged
cache that the verification step reads.

EfficientEdit (arXiv 2506.02780) Sec. III starts from a prompt -- the original
code and the instruction -- whose K/V the target model already holds.
``PromptIntake`` puts them there.  It owns the block table, the free list and
the lengths of B sequences on the device, and issues, on one stream:

    admit:   ee_prompt_slots          pages, positions and slots of the new tokens
    attend:  ee_rope_append           (each layer) rotary positions, K/V into the cache
             -> ee_prompt_attn        whole prompts, over their own K/V, or
             -> ee_chunk_attn         parts of prompts and single tokens, over the cache

Afterwards ``block_table``, ``ctx_len`` and the cache are what ``VerifyStep`` and
``EditSession`` take.  Those keep lengths of their own: ``commit`` hands back what
their steps committed (``EditSession.ctx_len``, ``VerifyStep.ctx_out``) before the
next ``admit``.  ``release`` takes a finished sequence's pages back.  The target
model's projections, which produce q, k and v, are the caller's.  No arithmetic on
them happens here; nothing is read back to the host.
"""
from __future__ import annotations

import math

import torch

from . import (EE_HEAD_DIM, EE_PAGE, ee_chunk_attn, ee_prompt_attn, ee_prompt_slots, ee_read_errors, ee_rope_append,
               new_prompt_workspace)


def rope_table(n_pos, base=1e6, device="cuda"):
    """ee_rope_append's table: [n_pos, 128] fp32, cosines of a position's 64 angles
    p base^(-i / 64), then sines; formed in 64 bits, once, at model load.  A model whose
    angles follow another rule (scaled positions, say) brings a table of that form."""
    half = EE_HEAD_DIM // 2
    inv = base ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * inv[None, :]
    return torch.cat((a.cos(), a.sin()), 1).float()


class PromptIntake:
    """Device-resident cache state of B sequences of one target model.

    k_cache / v_cache [L, num_pages, n_kv, 16, 128] bf16; rope fp32 [n_pos, 128]
    (``rope_table``).  max_pages: columns of the block table; max_tokens: new tokens
    of one call at most.  ``reserve`` positions after each sequence's new tokens get
    pages as well, as far as the table goes: room for the draft trees and commits of
    the steps until the next ``admit``, which gives it anew, also without new tokens.
    A ``VerifyStep`` in place takes the table itself, rather than a widened copy that
    later calls do not reach, when it has columns for max_ctx + max_T positions.  All
    pages are free at the start (``free_pages`` names others; ``release`` writes it).

    ``admit``, ``commit``, ``release`` and ``attend`` are capturable.  ``admit`` reads one of two
    sets of lengths and writes the other, so ``ctx_len`` is another tensor after each,
    and a graph that is to be replayed holds an even number of them."""

    def __init__(self, *, B, n_q, k_cache, v_cache, rope, max_pages, max_tokens, reserve=0, scale=None,
                 free_pages=None):
        if k_cache.dim() != 5 or k_cache.shape[3:] != (EE_PAGE, EE_HEAD_DIM) or v_cache.shape != k_cache.shape:
            raise ValueError("k_cache and v_cache must be [layers, pages, KV heads, 16, 128]")
        self.B, self.n_q, self.reserve = int(B), int(n_q), int(reserve)
        self.L, self.num_pages, self.n_kv = k_cache.shape[:3]
        self.k_cache, self.v_cache, self.rope = k_cache, v_cache, rope
        self.scale = 1.0 / math.sqrt(EE_HEAD_DIM) if scale is None else float(scale)
        dev = k_cache.device
        i32 = dict(dtype=torch.int32, device=dev)
        bf16 = dict(dtype=torch.bfloat16, device=dev)
        self.block_table = torch.full((self.B, int(max_pages)), -1, **i32)
        self.free_pages = torch.arange(self.num_pages, **i32) if free_pages is None else free_pages
        self._ctx = [torch.zeros(self.B, **i32) for _ in range(2)]
        self._held = [torch.zeros(self.B, **i32) for _ in range(2)]
        self._free = [torch.full((1,), self.free_pages.numel(), **i32) for _ in range(2)]
        self._now = 0                       # the current set of lengths
        self.tok_off = torch.zeros(self.B + 1, **i32)
        self._pos = torch.empty(int(max_tokens), **i32)
        self._slot = torch.empty(int(max_tokens), **i32)
        self._q = torch.empty((int(max_tokens), self.n_q, EE_HEAD_DIM), **bf16)
        self._k = torch.empty((int(max_tokens), self.n_kv, EE_HEAD_DIM), **bf16)
        self._out = torch.empty((int(max_tokens), self.n_q, EE_HEAD_DIM), **bf16)
        self.total = 0
        self.ws = new_prompt_workspace(device=dev)

    @property
    def ctx_len(self):
        """Tokens of each sequence, those of the last ``admit`` included (int32 [B])."""
        return self._ctx[self._now]

    @property
    def ctx_before(self):
        """Tokens of each sequence before the last ``admit`` (int32 [B])."""
        return self._ctx[self._now ^ 1]

    @property
    def held(self):
        """Pages each sequence holds: its block table's first columns (int32 [B])."""
        return self._held[self._now]

    @property
    def free_cnt(self):
        """Pages left: the first entries of ``free_pages`` (int32 [1])."""
        return self._free[self._now]

    def admit(self, new_len, total, stream=None):
        """Room for new_len[s] more tokens (device int32 [B]) of every sequence, ``total``
        in all (host): their order is ``tok_off``, and the layers' ``attend`` follow."""
        if not 0 <= total <= self._pos.numel():
            raise ValueError(f"total must lie in 0..{self._pos.numel()}")
        a, b = self._now, self._now ^ 1
        self.pos, self.slot = self._pos[:total], self._slot[:total]
        ee_prompt_slots(self._ctx[a], new_len, self._held[a], self.block_table, self.free_pages, self._free[a],
                        self.num_pages, self.reserve, self.tok_off, self.pos, self.slot, self._ctx[b], self._held[b],
                        self._free[b], self.ws, stream=stream)
        self.total, self._now = int(total), b

    def commit(self, ctx_len, stream=None):
        """The sequences' lengths after verification steps over the cache (device int32
        [B]): where the next ``admit`` goes on.  Copied; call it after the last admitted
        tokens' layers, which need the lengths before them."""
        if ctx_len.dtype is not torch.int32:
            raise TypeError(f"ctx_len must be {torch.int32}, got {ctx_len.dtype}")
        if ctx_len.shape != (self.B,) or not ctx_len.is_cuda:
            raise ValueError("ctx_len must be a CUDA tensor with an entry for each sequence")
        with torch.cuda.stream(stream):
            self.ctx_len.copy_(ctx_len)

    def release(self, done, stream=None):
        """Finished sequences (device bool [B]): their pages go to the end of the free list,
        in the table's order, their rows of the table to -1 and their lengths to zero; the
        next ``admit`` may give them a new prompt."""
        if done.dtype is not torch.bool:
            raise TypeError(f"done must be {torch.bool}, got {done.dtype}")
        if done.shape != (self.B,) or not done.is_cuda:
            raise ValueError("done must be a CUDA tensor with an entry for each sequence")
        with torch.cuda.stream(stream):
            n = self.free_pages.numel()
            gone = (torch.arange(self.block_table.shape[1], device=done.device) < self.held[:, None]) & done[:, None]
            at = self.free_cnt + gone.flatten().cumsum(0) - 1
            # an entry past the list takes what is not given back (and pages that never came from it)
            at = torch.where(gone.flatten(), at, n).clamp(0, n)
            free = torch.cat((self.free_pages, self.free_pages.new_empty(1)))
            self.free_pages.copy_(free.scatter_(0, at, self.block_table.flatten())[:n])
            self.free_cnt.add_(gone.sum()).clamp_(max=n)
            self.block_table.masked_fill_(done[:, None], -1)
            self.held.masked_fill_(done, 0)
            self.ctx_len.masked_fill_(done, 0)

    def attend(self, layer, q, k, v, whole=False, lse=None, stream=None):
        """Attention of the admitted tokens in one layer: q [total, n_q, 128], k and v
        [total, n_kv, 128] bf16 as projected (views of a fused projection's rows are
        taken as they are).  Writes K/V into the cache and returns [total, n_q, 128],
        valid until the next call; ``q_rot`` are the rotated queries.  ``whole``: no
        sequence had tokens before, so the new ones are all that they attend to."""
        n = self.total
        out, self.q_rot = self._out[:n], self._q[:n]
        kc, vc = self.k_cache[layer], self.v_cache[layer]
        k_rot = self._k[:n] if whole else None
        ee_rope_append(q, k, v, self.rope, self.pos, self.slot, self.q_rot, kc, vc, self.ws, k_out=k_rot,
                       stream=stream)
        if whole:
            ee_prompt_attn(self.q_rot, k_rot, v, self.tok_off, self.scale, out, self.ws, lse=lse, stream=stream)
        else:
            ee_chunk_attn(self.q_rot, kc, vc, self.block_table, self.ctx_before, self.tok_off, self.scale, out,
                          self.ws, lse=lse, stream=stream)
        return out

    def errors(self, stream=None):
        """Synchronise, return and clear the device error word (0 = none)."""
        return ee_read_errors(self.ws, stream=stream)
