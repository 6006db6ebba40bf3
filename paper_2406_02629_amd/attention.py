"""The attention of a transformer block on Shamir shares, from the block's input to the projection of its heads, with its keys and values
in a paged cache:

    share the input (GEN) -> queries, keys and values in one dense layer -> degree reduction, truncation -> rotary positions of the
    queries, keys (turned on the way) and values into the cache -> attention over the cache -> degree reduction, truncation -> dense
    layer of the heads -> degree reduction, truncation

With adapters, either dense layer adds each sequence's own low-rank change to its product, in front of the reduction.  Everything runs on the
shares; the result is a degree-t sharing at scale 2^f.  `Sequences` is the caller's side of the paged cache: which
pages belong to which sequence.
"""
from __future__ import annotations

from typing import Dict, List, Optional

import torch

from . import fixedpoint as fx
from .binding import Adapters, PagedCache, SSNet


class Sequences:
    """Pages of a cache, given to sequences as they grow."""

    def __init__(self, cache: PagedCache):
        self.cache = cache
        self.free: List[int] = list(range(cache.pages - 1, -1, -1))
        self.pages: Dict[int, List[int]] = {}
        self.length: Dict[int, int] = {}

    def release(self, name: int):
        """the sequence is over: its pages are free again"""
        self.free += reversed(self.pages.pop(name, []))
        self.length.pop(name, None)

    def extend(self, counts: Dict[int, int], device=None):
        """counts: new tokens of each sequence, in the order in which they stand in the batch.  Takes the pages that they need and
        returns what the calls ask for: dict(pos, slots, seq_start, block_table, ctx_len, max_ctx)."""
        batch, after = self.place(counts, device)
        self.keep(after)
        return batch

    def keep(self, after):
        """the second part of what place() returned: its tokens are in the cache"""
        sequences, taken = after
        del self.free[len(self.free) - taken:]
        for s, (pages, length) in sequences.items():
            self.pages[s], self.length[s] = pages, length

    def place(self, counts: Dict[int, int], device=None):
        """What extend() returns, and what keep() makes of the sequences once the calls have been made: until then they stay as they are, also
        if a call fails."""
        if any(c < 0 for c in counts.values()):
            raise ValueError("a sequence grows by no tokens or more")
        size = self.cache.page_size
        need = sum(-(-(self.length.get(s, 0) + c) // size) - len(self.pages.get(s, ())) for s, c in counts.items())
        if need > len(self.free):
            raise MemoryError(f"{need} pages needed, {len(self.free)} free")
        pos, slots, start, after, taken = [], [], [0], {}, 0
        for s, c in counts.items():
            pages, old = list(self.pages.get(s, ())), self.length.get(s, 0)
            while len(pages) * size < old + c:
                taken += 1
                pages.append(self.free[-taken])
            after[s] = pages, old + c
            pos += range(old, old + c)
            slots += [pages[p // size] * size + p % size for p in range(old, old + c)]
            start.append(start[-1] + c)
        longest = max(1, max(len(pages) for pages, _ in after.values()))
        table = [pages + [0] * (longest - len(pages)) for pages, _ in after.values()]
        lengths = [length for _, length in after.values()]

        def i32(v):
            return torch.tensor(v, dtype=torch.int32, device=device)

        return dict(pos=i32(pos), slots=torch.tensor(slots, dtype=torch.int64, device=device), seq_start=i32(start), block_table=i32(table),
                    ctx_len=i32(lengths), max_ctx=max(1, max(lengths))), (after, taken)


class Attention:
    """One attention layer.  w_qkv [width][(heads + 2 kv_heads) head_dim], w_out [heads head_dim][width]: float64 weights of the model's
    owner, shared and packed once.  table: fixedpoint.rotary_table.  weight_bits: f, or 2 f for long contexts (the weights of `length`
    keys are about 1 / length); default: what the longest context that table and cache have room for needs.  stream_base: the first
    stream id of its calls, each of which takes STREAMS of them; the two in front of it share the weights.  Default: whatever ids the context has free
    (SSNet.take_streams); ids that another layer has are refused.  adapters_qkv, adapters_out: sets of low-rank adapters of the two
    dense layers (any factor of theirs in B), of which forward gives each sequence one; a pass with adapters takes STREAMS +
    ADAPTER_STREAMS ids."""

    STREAMS = 8      # stream ids that a forward pass uses
    ADAPTER_STREAMS = 2

    def __init__(self, ss: SSNet, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, table: torch.Tensor, pages: int,
                 page_size: int = 64, layout: str = "half", weight_bits: Optional[int] = None, stream_base: Optional[int] = None,
                 adapters_qkv: Optional[Adapters] = None, adapters_out: Optional[Adapters] = None):
        self.ss, self.heads, self.kv, self.table, self.layout = ss, heads, kv_heads, table, layout
        self.dim = w_out.shape[0] // heads
        self.width = w_out.shape[1]
        if weight_bits is None:
            weight_bits = ss.f if ss.short_weights_serve(min(table.shape[0], pages * page_size)) else 2 * ss.f
        self.bits = weight_bits
        if self.bits not in (ss.f, 2 * ss.f):
            raise ValueError("weight_bits must be f or 2 f: the result is brought back to scale by truncations by 2^f")
        if w_qkv.shape != (self.width, (heads + 2 * kv_heads) * self.dim):
            raise ValueError("w_qkv must be [width][(heads + 2 kv_heads) head_dim]")
        for name, held, shape in (("adapters_qkv", adapters_qkv, w_qkv.shape), ("adapters_out", adapters_out, w_out.shape)):
            if held is not None and (held.K, held.N) != tuple(shape):
                raise ValueError(f"{name} must be of a layer {tuple(shape)}")
        self.adapters_qkv, self.adapters_out = adapters_qkv, adapters_out
        self.stream = stream_base        # of the next call, where the caller has a say
        weights = ss.take_streams(2, None if stream_base is None else stream_base - 2)

        def packed(w, stream):
            return ss.pack_weights_linear(ss.share(fx.encode(w.to(ss.device), ss.f, ss.p).contiguous(), stream_id=stream))

        self.w_qkv, self.w_out = packed(w_qkv, weights + 1), packed(w_out, weights)
        self.cache = PagedCache(ss, pages, page_size, kv_heads, self.dim)
        self.sequences = Sequences(self.cache)

    def forward(self, x: torch.Tensor, counts: Dict[int, int], adapters: Optional[Dict[int, int]] = None) -> torch.Tensor:
        """x: shares [n][tokens][width] at scale 2^f of the new tokens, counts as in Sequences.extend -> shares [n][tokens][width].  adapters: the place in the
        layer's sets that a sequence's adapter has (a set that ends before it changes nothing); sequences that are not in it, or at -1, have none.  A call
        that is refused or fails leaves the sequences as they were."""
        ss, heads, kv, dim = self.ss, self.heads, self.kv, self.dim
        n, tokens, _ = x.shape
        if sum(counts.values()) != tokens:
            raise ValueError("counts must add up to the tokens of x")
        batch, after = self.sequences.place(counts, x.device)
        if batch["max_ctx"] > self.table.shape[0]:
            raise ValueError(f"the table has {self.table.shape[0]} positions, a sequence would have {batch['max_ctx']}")
        index = None
        if adapters is not None:
            if self.adapters_qkv is None and self.adapters_out is None:
                raise ValueError("the layer has no adapters")
            places, held = [adapters.get(s, -1) for s in counts], max(a.adapters for a in (self.adapters_qkv, self.adapters_out) if a is not None)
            if not all(-1 <= i < held for i in places):
                raise ValueError(f"a sequence's adapter must be a place of the layer's sets, 0 to {held - 1}, or -1: {places}")
            index = torch.tensor(places, dtype=torch.int32, device=x.device)
        streams = self.STREAMS + (self.ADAPTER_STREAMS if adapters is not None else 0)
        stream = ss.take_streams(streams, self.stream)
        if self.stream is not None:
            self.stream += streams

        def adapted(held, x, y, own):
            return y if held is None or index is None else ss.adapters_mod(held, x, batch["seq_start"], index, own, base=y, out=y)

        qkv = adapted(self.adapters_qkv, x, ss.linear_mod_packed(x, self.w_qkv, (heads + 2 * kv) * dim), stream + self.STREAMS)
        qkv = ss.degree_reduce_truncate(qkv, stream_id=stream).view(n, tokens, heads + 2 * kv, dim)
        q = ss.rotary_truncate(qkv[:, :, :heads], self.table, batch["pos"], stream + 1, layout=self.layout)
        ss.cache_append(self.cache, qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:], batch["slots"], stream + 2, table=self.table,
                        pos=batch["pos"], layout=self.layout)
        o = ss.paged_attention(self.cache, q, batch["seq_start"], batch["block_table"], batch["ctx_len"], batch["max_ctx"], stream + 3,
                               weight_bits=self.bits)
        o = ss.degree_reduce_truncate(o, stream_id=stream + 4)
        if self.bits == 2 * ss.f:
            o = ss.truncate(o, stream_id=stream + 5)
        o = o.view(n, tokens, heads * dim)
        y = adapted(self.adapters_out, o, ss.linear_mod_packed(o, self.w_out, self.width), stream + self.STREAMS + 1)
        y = ss.degree_reduce_truncate(y, stream_id=stream + 6)
        self.sequences.keep(after)
        return y
