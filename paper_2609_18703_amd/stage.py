"""The attention of a model stage on the batches that the framework forms.

A stage runs on a reservation of ro_batch: B children, parents mixed.  Every
child is one sequence over a paged cache: it reads its parent's prompt, which
lies in pages that all siblings name, and then its own pages, the first of
which has what the prompt leaves in a page that it does not fill.  The tables
that say so come from the batch's tags, on the device: nothing here waits for
them.

The functions only sequence library calls on device tensors, all on the
context's stream, whichever is torch's current one: inputs have to be ready
there, and outputs are.  One layer is shown; a model's layers share the plan
and have a cache each.

    stage = Stage(ctx, parents, children, ...)
    stage.prompts(qkv, pos, q_off, lengths)  # once: every parent's prompt enters its pages
    stage.reserve(out_child, out_parent)     # a batch's children become the sequences
    out = stage.step(qkv, pos, q_off, new)   # their next tokens, as often as needed
    stage.shrink(budget, first, last)        # where caches outgrow their room
"""
from __future__ import annotations

import functools

import torch

from .ro import Cache, Rotary

__all__ = ["Stage"]

NO_PAGE = -1        # no cache has this page: positions in it are an error, and nothing is written to them


def _on_stream(f):
    """Runs a method's own work on tensors where its library calls run."""
    @functools.wraps(f)
    def run(self, *args, **kw):
        with torch.cuda.stream(self.ctx._stream):
            return f(self, *args, **kw)
    return run


class Stage:
    def __init__(self, ctx, n_parents, n_children, batch, q_heads, kv_heads, head_dim, page_size, prompt_pages,
                 child_pages, rotary: Rotary, max_new, dtype=torch.bfloat16, window=0, sinks=0):
        self.ctx, self.rotary, self.window, self.sinks = ctx, rotary, window, sinks
        self._make(n_parents, n_children, batch, q_heads, kv_heads, head_dim, page_size, prompt_pages, child_pages,
                   max_new, dtype)

    @_on_stream
    def _make(self, n_parents, n_children, batch, q_heads, kv_heads, head_dim, page_size, prompt_pages, child_pages,
              max_new, dtype):
        ctx = self.ctx
        self.P, self.N, self.B = int(n_parents), int(n_children), int(batch)
        self.Hq, self.Hk, self.D, self.ps = q_heads, kv_heads, head_dim, page_size
        self.prompt_pages, self.child_pages, self.max_new = prompt_pages, child_pages, int(max_new)
        # pages: the parents' prompts, the children's own, and a batch's shrunk caches
        most = prompt_pages + child_pages
        self.own0 = self.P * prompt_pages
        self.kept0 = self.own0 + self.N * child_pages
        shape = (self.kept0 + 2 * self.B * most, kv_heads, page_size, head_dim)
        dev = dict(dtype=dtype, device="cuda")
        self.cache = Cache(torch.zeros(shape, **dev), torch.zeros(shape, **dev))
        self.parents = ctx.chunk(self.P, self.P * prompt_pages * page_size, prompt_pages)
        self.chunk = ctx.chunk(self.B, self.B * self.max_new, most)
        self.table = torch.zeros(0, most, dtype=torch.int32, device="cuda")
        # two sets of pages in turn: what is kept never goes to pages that it comes from
        self.kept = list((self.kept0 + torch.arange(2 * self.B * most, device="cuda")).int().view(2, self.B, most))
        self.n = 0                                # sequences: children of the present reservation
        self.planned = False                      # does the plan hold their present lengths and pages?
        self.kv_len = torch.zeros(0, dtype=torch.int32, device="cuda")
        self.prompt_len = torch.zeros(self.P, dtype=torch.int32, device="cuda")
        self.weight = torch.zeros(self.B, most * page_size, device="cuda")

    def _layer(self, chunk, qkv, pos):
        Hq, Hk = self.Hq, self.Hk
        q = torch.empty(qkv.shape[0], Hq, self.D, dtype=qkv.dtype, device="cuda")
        lse = torch.empty(qkv.shape[0], Hq, device="cuda")
        chunk.append(self.cache, qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], q, self.rotary, pos)
        out = torch.empty_like(q)
        chunk.attend(self.cache, q, out, lse)
        return q, out, lse

    @_on_stream
    def prompts(self, qkv, pos, q_off, lengths):
        """Every parent's prompt: qkv [tokens, q heads + 2 kv heads, dim], q_off [P + 1], lengths [P] (int32)."""
        pages = torch.arange(self.P * self.prompt_pages, device="cuda").int().view(self.P, self.prompt_pages)
        # (a length that its pages do not hold is the plan's error, and an empty prompt)
        held = (lengths >= 0) & (lengths <= self.prompt_pages * self.ps)
        self.prompt_len.copy_(torch.where(held, lengths, 0))
        self.parents.plan(self.cache, q_off, lengths, pages, self.Hq, n_tokens=qkv.shape[0],
                          max_new=self.prompt_pages * self.ps, window=self.window, sinks=self.sinks)
        return self._layer(self.parents, qkv, pos)[1]

    @_on_stream
    def reserve(self, out_child, out_parent):
        """The children of a reservation (the batch's tags, on the device: up to as many as the stage was made for,
        fewer in a last reservation that is not full) are the sequences from now on."""
        self.n = min(self.B, out_child.numel())
        child, parent = out_child[:self.n].long(), out_parent[:self.n].long()
        self.kv_len = self.prompt_len[parent]
        # a parent's prompt pages, as many as it fills, then the child's own, then none
        col = torch.arange(self.table.shape[1], device="cuda")
        have = (self.kv_len // self.ps)[:, None]
        prompt = parent[:, None] * self.prompt_pages + col
        own = self.own0 + child[:, None] * self.child_pages + (col - have)
        self.table = torch.where(col < have, prompt, torch.where(col < have + self.child_pages, own, NO_PAGE)).int()
        # a prompt that ends inside a page: the child goes on in a copy of it, the first of its own
        if self.prompt_pages and self.child_pages:
            end = parent * self.prompt_pages + have[:, 0].clamp(max=self.prompt_pages - 1)
            for pages in (self.cache.k, self.cache.v):
                pages[self.own0 + child * self.child_pages] = pages[end]
        self.weight.zero_()
        self.planned = False

    def _plan(self, q_off, n_tokens, kv_len):
        self.planned = False                      # until the call that needs it has been taken
        self.chunk.plan(self.cache, q_off, kv_len, self.table, self.Hq, n_tokens=n_tokens,
                        max_new=min(self.max_new, n_tokens), window=self.window, sinks=self.sinks)

    @_on_stream
    def step(self, qkv, pos, q_off, new):
        """The next tokens of every sequence (new [seqs] int32, q_off [seqs + 1]): appended, attended, weighed."""
        kv_len = self.kv_len + new
        self._plan(q_off, qkv.shape[0], kv_len)
        q, out, lse = self._layer(self.chunk, qkv, pos)
        self.kv_len, self.planned = kv_len, True
        weight = self.weight[:self.n]
        self.chunk.weigh(self.cache, q, lse, weight, weight)
        return out

    @_on_stream
    def shrink(self, budget, first, last):
        """Keep `budget` positions of every sequence, in pages of the batch's own; index [seqs, budget] of the kept ones."""
        if not self.planned:                      # right after a reservation, or after another eviction
            self._plan(torch.zeros(self.n + 1, dtype=torch.int64, device="cuda"), 0, self.kv_len)
        index = torch.empty(self.n, budget, dtype=torch.int32, device="cuda")
        weight = torch.zeros(self.n, budget, device="cuda")
        kv_len, table = torch.empty_like(self.kv_len), self.kept[1][:self.n]
        self.chunk.evict(self.cache, self.weight, table, budget, kv_len, index, weight, first=first, last=last)
        self.kv_len, self.table = kv_len, table
        self.kept.reverse()
        cols = min(budget, self.weight.shape[1])
        self.weight.zero_()
        self.weight[:self.n, :cols] = weight[:, :cols]
        self.planned = False
        return index
