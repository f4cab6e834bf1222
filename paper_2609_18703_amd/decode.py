"""Tokens of a batch's children, one step after another, over a pool of pages.

A reservation's children share their parents' prompts: forking copies rows of
page numbers, not pages.  Every step takes the room that its tokens need, a
page of the sequence's own where it shares a partly filled one, projects the
tokens through 8-bit weights, attends over the pages, and may choose the next
token from the logits.  Sequences that have ended give their pages back, and
a pool that is full of holes is compacted.  Lengths, tables and counts stay
on the device: nothing here waits for them.

The functions only sequence library calls, all on the context's stream,
whichever is torch's current one: inputs have to be ready there, and outputs
are.  The layers are attention alone: x + out(attend(qkv(x))).

    decode = Decode(ctx, parents, children, layers, ...)
    decode.prompts(x, pos, q_off, lengths)        # once: every parent's prompt
    decode.reserve(out_child, out_parent)         # a batch's children in place of the last one's
    h = decode.step(x, pos, q_off, new)           # their next tokens, as often as needed
    token, logprob = decode.choose(h[last], u, temperature=...)
    decode.keep(lengths)                          # 0 for those that have ended
    decode.compact()
"""
from __future__ import annotations

import torch

from .ro import ECAP, NO_PAGE, Cache, RoError, Rotary, Tables, Weights, _pos, _ptr, _typed
from .stage import _on_stream

__all__ = ["Decode", "Projection"]


class Projection:
    """A product with 8-bit weights, of rows that become 8-bit integers on the way."""

    def __init__(self, ctx, weights: Weights):
        self.ctx, self.weights = ctx, weights

    def __call__(self, x, dtype=None):
        q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
        scale = torch.empty(x.shape[0], device="cuda")
        out = torch.empty(x.shape[0], self.weights.n_out, dtype=dtype or x.dtype, device="cuda")
        self.ctx.quantize(x, q, scale)
        self.ctx.project(q, scale, self.weights, out)
        return out


class Decode:
    """layers: a pair of Weights each, to queries, keys and values [(q heads + 2 kv heads) * dim, hidden] and back
    [hidden, q heads * dim]; head: Weights to logits, or None."""

    def __init__(self, ctx, n_parents, batch, layers, head, q_heads, kv_heads, head_dim, page_size, n_pages, max_pages,
                 rotary: Rotary, max_tokens, dtype=torch.bfloat16):
        self.ctx, self.rotary, self.dtype = ctx, rotary, dtype
        self.P, self.B = int(n_parents), int(batch)
        self.Hq, self.Hk, self.D, self.max_tokens = q_heads, kv_heads, head_dim, int(max_tokens)
        self.layers = [(Projection(ctx, a), Projection(ctx, b)) for a, b in layers]
        self.head = None if head is None else Projection(ctx, head)
        for a, b in layers:
            sizes = a.n_out, b.n_in, a.n_in, b.n_out
            hidden = layers[0][0].n_in
            if sizes != ((q_heads + 2 * kv_heads) * head_dim, q_heads * head_dim, hidden, hidden):
                raise ValueError(f"a layer's weights are [{sizes[0]}, {sizes[2]}] and [{sizes[3]}, {sizes[1]}]: not those of "
                                 f"{q_heads} and {kv_heads} heads of {head_dim} beside {hidden} channels")
        if head is not None and layers and head.n_in != layers[0][0].n_in:
            raise ValueError(f"the head takes {head.n_in} channels, the layers have {layers[0][0].n_in}")
        self._make(n_pages, max_pages, page_size)

    @_on_stream
    def _make(self, n_pages, max_pages, page_size):
        dev = dict(dtype=self.dtype, device="cuda")
        shape = (n_pages, self.Hk, page_size, self.D)
        self.caches = [Cache(torch.zeros(shape, **dev), torch.zeros(shape, **dev)) for _ in self.layers]
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        rows = max(self.P, self.B)
        self.pool = self.ctx.pages(self.refs, page_size, rows)
        self.chunk = self.ctx.chunk(rows, self.max_tokens, max_pages)
        self.parents, self.children = (
            Tables(torch.full((n, max_pages), NO_PAGE, dtype=torch.int32, device="cuda"),
                   torch.zeros(n, dtype=torch.int32, device="cuda")) for n in (self.P, self.B))
        self.moved = [torch.empty(max(rows, n_pages // 2), dtype=torch.int32, device="cuda") for _ in range(3)]
        self.moves = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.n_free = torch.zeros(1, dtype=torch.int64, device="cuda")
        if self.layers:
            # (a step without tokens: heads, pages and rotations that the library does not take are refused here)
            none = self.parents.len
            self.chunk.plan(self.caches[0], torch.zeros(self.P + 1, dtype=torch.int64, device="cuda"), none,
                            self.parents.table, self.Hq, n_tokens=0)
            rows = torch.empty(0, self.Hq + 2 * self.Hk, self.D, **dev)
            q, k, v = rows.split([self.Hq, self.Hk, self.Hk], 1)
            axes = self.rotary.n_axes if self.rotary else 1
            self.chunk.append(self.caches[0], q, k, v, torch.empty_like(q), self.rotary,
                              torch.empty(axes, 0, dtype=torch.int32, device="cuda"))

    def _run(self, tables, x, pos, q_off, new):
        n = tables.n_seqs
        # what a call below would refuse is refused before the pool changes, the tokens by the first projection
        if x.dtype is not self.dtype:
            raise TypeError(f"tokens need {self.dtype}, have {x.dtype}")
        T = x.shape[0]
        if T > self.max_tokens:
            raise RoError(ECAP, f"a step of {T} tokens, {self.max_tokens} at most")
        _ptr(q_off, 8, n + 1, "q_off")
        _typed(new, "int32", n, "new")
        _pos(pos, self.rotary, T)
        first = self.layers[0][0](x) if self.layers else None
        src, dst, slots = (t[:n] for t in self.moved)
        want = tables.len + new
        self.pool.grow(tables, new, src, dst, slots, self.n_free)
        # (a sequence that got no room is none: its tokens have no place that is its own)
        length = torch.where(tables.len == want, want, -1)
        self.pool.copy(self.caches, src, dst, slots)
        Hq, Hk, D = self.Hq, self.Hk, self.D
        for i, (qkv, back) in enumerate(self.layers):
            if i == 0:
                self.chunk.plan(self.caches[0], q_off, length, tables.table, Hq, n_tokens=T)
            rows = (qkv(x) if i else first).view(T, Hq + 2 * Hk, D)
            q = torch.empty(T, Hq, D, dtype=self.dtype, device="cuda")
            self.chunk.append(self.caches[i], rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:], q, self.rotary, pos)
            out = torch.empty_like(q)
            self.chunk.attend(self.caches[i], q, out)
            x = x + back(out.view(T, Hq * D))
        return x

    @_on_stream
    def prompts(self, x, pos, q_off, lengths):
        """Every parent's prompt: x [tokens, hidden], pos [axes, tokens], q_off [P + 1], lengths [P] (int32)."""
        return self._run(self.parents, x, pos, q_off, lengths)

    @_on_stream
    def reserve(self, out_child, out_parent):
        """The children of a reservation (the batch's tags, on the device; fewer than the batch in one that is not
        full) are the sequences from now on, each with its parent's prompt."""
        n = min(self.B, out_child.numel())
        if out_parent.numel() < n:
            raise ValueError(f"{n} children, {out_parent.numel()} parents")
        parent = torch.full((self.B,), -1, dtype=torch.int32, device="cuda")
        parent[:n] = out_parent[:n]
        self.pool.release(self.children)
        self.pool.fork(self.parents, parent, self.children)

    @_on_stream
    def step(self, x, pos, q_off, new):
        """The next tokens of every sequence: x [tokens, hidden], q_off [batch + 1], new [batch] (int32, 0 for rows
        without a child).  Where the pool has too few pages for all (RO_ECAP in the context's status), the sequences
        and the pages stay as they were, and what is returned means nothing.  So do they where a call is refused."""
        return self._run(self.children, x, pos, q_off, new)

    @_on_stream
    def choose(self, hidden, u, **how):
        """A token and its log-probability for every row of hidden (filters as in Context.sample)."""
        token = torch.empty(hidden.shape[0], dtype=torch.int32, device="cuda")
        logprob = torch.empty(hidden.shape[0], device="cuda")
        self.ctx.sample(self.head(hidden), u, token, logprob, **how)
        return token, logprob

    @_on_stream
    def keep(self, lengths):
        """Sequences keep their first lengths [batch] (int32) positions: 0 for those that have ended, fewer than they
        have where tokens are taken back."""
        self.pool.release(self.children, lengths)

    @_on_stream
    def compact(self):
        """The pages in use become the first ones of the pool."""
        src, dst, _ = self.moved
        self.pool.compact([self.parents, self.children], src, dst, self.moves, self.n_free)
        self.pool.copy(self.caches, src, dst, n=self.moves)
