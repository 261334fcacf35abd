"""What a destination does with the requests that are routed to it: a small server over the prefix-cache calls.

The router sends requests of one key to destinations that hold the key's prefix (paper sec. 3.2).  ``Destination`` keeps
those prefixes in pages of a key/value cache, one table row each:

  admit   prefixes that are not held are read into pages (whole prompts, ``attn_paged``), idle ones leaving, least
          recent first, when rows or pages run out; every request forks its key's prefix, gets pages for its own tokens, writes their keys and
          values and attends over prefix and suffix;
  step    one more token for every running request; requests of one key stand together, so that their prefix is read
          once for all of them (``attn_decode``);
  finish  rows of finished requests become empty; ``compact`` moves live pages to the front.

The model is the caller's: ``layers``, ``embed(tokens) -> x``, ``qkv(layer, x) -> q, k, v`` ([tokens, heads, head_dim])
and ``mix(layer, x, out) -> x``.  Bookkeeping of rows is on the host; nothing here waits for the GPU.

Every call runs on the context's stream, the model's passes among it: after what torch's current stream has when the
call is made, and before what that stream gets next.
"""
from __future__ import annotations

import functools
from collections import OrderedDict
from typing import Dict, List, Sequence, Tuple

from . import (Context, KVPages, attn_decode, attn_paged, kv_write, pages_compact, pages_extend, pages_fork,
               pages_free)


def _on_context_stream(call):
    """The call's work on the context's stream, in the current stream's order.  Lists and results are allocated there: a
    list that is dropped is not handed out again before the kernels that read it."""
    @functools.wraps(call)
    def ordered(self, *args, **kw):
        if not self.pages.lens.is_cuda:
            return call(self, *args, **kw)
        import torch
        mine, here = self.ctx.stream, torch.cuda.current_stream(self.pages.lens.device)
        if mine.cuda_stream == here.cuda_stream:
            return call(self, *args, **kw)
        mine.wait_stream(here)
        _used_on((args, list(kw.values())), mine)
        try:
            with torch.cuda.stream(mine):
                result = call(self, *args, **kw)
            _used_on((result, self.pages.ref, self.pages.table), here)
            return result
        finally:
            here.wait_stream(mine)
    return ordered


def _used_on(values, stream):
    """Tensors among the values are not handed out again before ``stream`` has passed their last use."""
    for v in values:
        if isinstance(v, (tuple, list)):
            _used_on(v, stream)
        elif getattr(v, "is_cuda", False):
            v.record_stream(stream)


class Destination:
    def __init__(self, ctx: Context, pages: KVPages, model):
        self.ctx, self.pages, self.model = ctx, pages, model
        self.free_rows: List[int] = list(range(pages.lens.shape[0]))[::-1]
        self.free_pages = pages.n_pages
        self.prefixes: "OrderedDict[int, Tuple[int, int]]" = OrderedDict()  # key -> (row, tokens), least recent first
        self.running: "OrderedDict[int, List[int]]" = OrderedDict()         # key -> rows of its running requests
        self.own: Dict[int, Tuple[int, int]] = {}                           # row -> (tokens, pages that are its alone)
        self.kept: Dict[int, int] = {}                                      # running row -> tokens of its key's prefix

    def _ints(self, values):
        import torch
        lens = self.pages.lens
        if not lens.is_cuda:
            return torch.tensor(list(values), dtype=torch.int32)
        # from pinned memory, which torch keeps until the copy has passed: one from pageable memory waits for the stream
        return torch.tensor(list(values), dtype=torch.int32, pin_memory=True).to(lens.device, non_blocking=True)

    def _cu(self, lens):
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        return self._ints(at)

    def _check_width(self, tokens: int) -> None:
        """A row that cannot hold its tokens is not grown by the library, and what is then written goes to other places."""
        width = self.pages.table.shape[1] * self.pages.page
        if tokens > width:
            raise RuntimeError(f"a row of {width} tokens has no room for {tokens}")

    def _pages(self, tokens: int) -> int:
        return -(-tokens // self.pages.page)

    def _forward(self, tokens, cu, rows, groups=None):
        """One pass of the model, without gradients, over new tokens that the rows' lengths already count."""
        import torch
        with torch.no_grad():
            x = self.model.embed(tokens)
            for layer in range(self.model.layers):
                q, k, v = self.model.qkv(layer, x)
                kv_write(self.ctx, self.pages, layer, k, v, cu, seqs=rows)
                if groups is None:
                    out = attn_paged(self.ctx, q, self.pages, layer, cu, seqs=rows)
                else:
                    out = attn_decode(self.ctx, q, self.pages, layer, seqs=rows, group_off=groups[0], shared=groups[1])
                x = self.model.mix(layer, x, out)
            return x

    def _make_room(self, rows: int, pages: int, keep) -> None:
        """Idle prefixes leave, least recent first, until rows and pages are free; nothing changes if that is too few."""
        gone, r, p = [], len(self.free_rows), self.free_pages
        for key, (row, _) in self.prefixes.items():
            if r >= rows and p >= pages:
                break
            if not self.running.get(key) and key not in keep:
                gone.append(key)
                r, p = r + 1, p + self.own[row][1]
        if r < rows or p < pages:
            raise RuntimeError(f"a destination of {self.pages.lens.shape[0]} rows and {self.pages.n_pages} pages has no "
                               f"room for {rows} rows and {pages} pages more")
        if gone:
            self._free([self.prefixes.pop(key)[0] for key in gone])

    def _take(self, tokens: int, pages: int) -> int:
        row = self.free_rows.pop()
        self.own[row] = (tokens, pages)
        self.free_pages -= pages
        return row

    def _free(self, rows: Sequence[int]) -> None:
        pages_free(self.ctx, self.pages, self._ints(rows))
        for row in rows:
            self.free_pages += self.own.pop(row)[1]
            self.kept.pop(row, None)
        self.free_rows.extend(rows)

    @_on_context_stream
    def admit(self, requests: Sequence[Tuple[int, object, int]]):
        """requests: (key, tokens, prefix length).  Requests of a key may keep less of its prefix than is held (a prefix
        that is not held is read as far as the longest of the call keeps it), not more.  Returns each request's row and
        the model's output for its own tokens, back to back.  If the model or a call fails, the call's requests and the
        prefixes that it was to read are given up."""
        import torch
        page = self.pages.page
        if not requests:
            raise ValueError("no requests")
        new: Dict[int, object] = {}
        for key, tokens, plen in requests:
            if not 1 <= plen <= int(tokens.shape[0]):
                raise ValueError(f"a prefix of {plen} tokens in a prompt of {int(tokens.shape[0])}")
            if key in self.prefixes:
                if plen > self.prefixes[key][1]:
                    raise ValueError(f"key {key} is held with a prefix of {self.prefixes[key][1]} tokens, not {plen}")
            elif key not in new or plen > new[key].shape[0]:
                new[key] = tokens[:plen]
        own = [tokens[plen:] for _, tokens, plen in requests]
        whole = [int(tokens.shape[0]) for _, tokens, _ in requests]
        self._check_width(max(whole))
        alone = [self._pages(n) - plen // page for n, (_, _, plen) in zip(whole, requests)]
        self._make_room(len(new) + len(requests),
                        sum(self._pages(int(t.shape[0])) for t in new.values()) + sum(alone),
                        {key for key, _, _ in requests})
        taken: List[int] = []
        try:
            if new:
                lens = [int(t.shape[0]) for t in new.values()]
                for key, n in zip(new, lens):
                    taken.append(self._take(n, self._pages(n)))
                    self.prefixes[key] = (taken[-1], n)
                rows = self._ints(taken)
                pages_extend(self.ctx, self.pages, rows, self._ints(lens))
                self._forward(torch.cat(list(new.values())), self._cu(lens), rows)
            rows = [self._take(n, p) for n, p in zip(whole, alone)]
            taken += rows
            for (key, _, plen), row in zip(requests, rows):
                self.prefixes.move_to_end(key)
                self.running.setdefault(key, []).append(row)
                self.kept[row] = plen
            dst, lens = self._ints(rows), [int(t.shape[0]) for t in own]
            pages_fork(self.ctx, self.pages, self._ints(self.prefixes[key][0] for key, _, _ in requests), dst,
                       self._ints(plen for _, _, plen in requests))
            pages_extend(self.ctx, self.pages, dst, self._ints(lens))
            return rows, self._forward(torch.cat(own), self._cu(lens), dst)
        except BaseException:
            self._give_up(taken)
            raise

    def _give_up(self, rows: Sequence[int]) -> None:
        """Rows whose keys and values were not all written leave, prefixes among them."""
        gone = set(rows)
        for key in [key for key, (row, _) in self.prefixes.items() if row in gone]:
            del self.prefixes[key]
        self._leave(gone)
        if gone:
            self._free(list(rows))

    def _leave(self, gone) -> None:
        for key in list(self.running):
            self.running[key] = [row for row in self.running[key] if row not in gone]
            if not self.running[key]:
                del self.running[key]

    def order(self) -> List[int]:
        """Rows of the running requests as ``step`` takes them."""
        return [row for rows in self.running.values() for row in rows]

    @_on_context_stream
    def step(self, tokens):
        """One more token for every running request, in ``order()``: the model's output [requests, ...].  If the model or
        a call fails, the running requests are given up: their last token's keys and values are not in every layer."""
        rows, page = self.order(), self.pages.page
        if len(tokens) != len(rows):
            raise ValueError(f"{len(tokens)} tokens for {len(rows)} running requests")
        self._check_width(max((self.own[row][0] + 1 for row in rows), default=0))
        grown = {row: (self.own[row][0] + 1, self.own[row][1] + (self.own[row][0] % page == 0)) for row in rows}
        more = sum(p - self.own[row][1] for row, (_, p) in grown.items())
        self._make_room(0, more, ())
        self.own.update(grown)
        self.free_pages -= more
        off, shared = [0], []
        for key, mine in self.running.items():
            if mine:
                off.append(off[-1] + len(mine))
                # whole pages that all of them kept: behind the shortest they are each request's own
                shared.append(min(self.kept[row] for row in mine) // page * page)
        try:
            r = self._ints(rows)
            pages_extend(self.ctx, self.pages, r, self._ints([1] * len(rows)))
            return self._forward(tokens, self._ints(range(len(rows) + 1)), r, (self._ints(off), self._ints(shared)))
        except BaseException:
            self._give_up(rows)
            raise

    @_on_context_stream
    def finish(self, rows: Sequence[int]) -> None:
        """Rows of requests that have ended become empty; their keys' prefixes stay."""
        gone = set(rows)
        if len(gone) != len(rows) or not gone.issubset(self.kept):
            raise ValueError(f"rows {list(rows)}: a running request's each, once")
        if not gone:
            return
        self._free(list(rows))
        self._leave(gone)

    @_on_context_stream
    def compact(self):
        """Live pages to the front of the pool; their number (on the device)."""
        ref, table, _, live = pages_compact(self.ctx, self.pages)
        self.pages.replace(ref, table)
        return live
