"""Who holds which page of a paged key-value cache.

Sec. 3.2 shortens a sequence's cache at every pruning layer; ``PagePool`` gives what that frees to other
sequences.  It keeps the page lists, reference counts and lengths of up to ``max_seqs`` sequences on the host,
mirrors them in the int32 page table and length tensors that the operators read, and calls ``apack_copy_pages``
and ``apack_paged_compact`` where pages have to move.  A fork shares its parent's pages; a page that is shared is
copied when a sequence first writes behind its last row.

All device work is queued on torch's current stream; a pool's calls belong on one stream (a page that is freed
may be handed out again by the next call) and are not captured (a graph reads the tables that they change).
Every method checks that it can be carried out (pages, rows) before it changes anything, and changes what the host
keeps only after its device calls have been queued: one that raises (an allocation, a pool on another device than
the current one) leaves every sequence as it was.
"""

import numpy as np
import torch

from . import PagedCache, apack_copy_pages, apack_paged_compact


class PagePool:
    """Pools ``k`` and ``v`` [layers, pages, page_tokens, Hkv, D], ``page_table`` [max_seqs, max_pages] and
    ``lengths`` [max_seqs] on the device, and ``cache``, the PagedCache of all of it.

    A sequence has one length and one list of pages for all layers.  Layers that keep different rows (the levels of
    a progressive schedule) take a pool each.

    heads_first: the heads of a page outermost in memory ([layers, pages, Hkv, page_tokens, D])."""

    def __init__(self, num_layers, num_pages, page_tokens, num_kv_heads, head_dim, max_seqs, max_pages=None,
                 dtype=torch.bfloat16, device="cuda", heads_first=False):
        max_pages = num_pages if max_pages is None else max_pages
        shape = (num_layers, num_pages, num_kv_heads, page_tokens, head_dim) if heads_first else (
            num_layers, num_pages, page_tokens, num_kv_heads, head_dim)
        self.k, self.v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        if heads_first:
            self.k, self.v = self.k.permute(0, 1, 3, 2, 4), self.v.permute(0, 1, 3, 2, 4)
        self.page_tokens, self.max_pages, self.device = page_tokens, max_pages, device
        self.page_table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self.cache = PagedCache(self.k, self.v, self.page_table)
        self._refs = np.zeros(num_pages, np.int64)
        self._free = list(range(num_pages - 1, -1, -1))
        self._pages = [None] * max_seqs          # page list of a sequence, None where the row is unused
        self._len = np.zeros(max_seqs, np.int64)  # ceil(length / page_tokens) pages are held
        self._shared = 0                         # sum over the pages of the holders beyond the first

    # ------------------------------------------------------------ host state

    @property
    def free_pages(self):
        return len(self._free)

    def length(self, seq):
        self._held(seq)
        return int(self._len[seq])

    def pages(self, seq):
        return list(self._held(seq))

    def _held(self, seq):
        if not 0 <= seq < len(self._pages) or self._pages[seq] is None:
            raise ValueError(f"sequence {seq} is not in the pool")
        return self._pages[seq]

    def _need(self, rows):
        n = -(-int(rows) // self.page_tokens)
        if rows < 0 or n > self.max_pages:
            raise ValueError(f"{rows} rows: 0 to {self.max_pages * self.page_tokens} fit a sequence")
        return n

    def _room(self, pages, seqs=0):
        if pages > len(self._free):
            raise MemoryError(f"{pages} pages wanted, {len(self._free)} free")
        rows = [i for i, p in enumerate(self._pages) if p is None]
        if seqs > len(rows):
            raise MemoryError(f"{seqs} sequences wanted, {len(rows)} rows of the page table free")
        return rows[:seqs]

    def _spare(self, n):
        """The pages that the next _take(n) takes."""
        return self._free[len(self._free) - n:][::-1]

    def _take(self, n):
        got = self._spare(n)
        del self._free[len(self._free) - n:]
        self._refs[got] = 1

    def _drop(self, pages):
        at = np.asarray(pages, np.int64)         # distinct
        self._refs[at] -= 1
        gone = at[self._refs[at] == 0]
        self._free += gone.tolist()
        self._shared -= len(at) - len(gone)

    def _device(self, values):
        """An array on the device, without waiting for the stream: through pinned memory, which torch does not hand
        out again before it has been read."""
        host = torch.from_numpy(values)
        return (host.pin_memory() if self.k.is_cuda else host).to(self.device, non_blocking=True)

    def _stage(self, at, length, entries, more=()):
        """What _write needs of an update, on the device; nothing is changed.  Lengths of the sequences `at` and, pairs of
        (place in the flat table, page), their entries; `more` for the caller.  One copy for all of them."""
        n, m = len(at), len(entries)
        both = np.array(entries, np.int64).reshape(m, 2)
        wide = self._device(np.concatenate([at, both[:, 0], length, both[:, 1], more]).astype(np.int64))
        return n, m, wide, wide[n + m:].to(torch.int32)

    def _stage_rows(self, seqs, lists, length):
        """The same for these sequences' whole rows."""
        return self._stage(np.asarray(seqs, np.int64), length,
                           [(s * self.max_pages + i, p) for s, pages in zip(seqs, lists) for i, p in enumerate(pages)])

    def _write(self, staged, clear=False):
        """A staged update of the device's tables; returns its `more`.  clear: -1 in all other entries of the sequences."""
        n, m, wide, narrow = staged
        if clear:
            self.page_table.index_fill_(0, wide[:n], -1)
        if m:
            self.page_table.view(-1).index_copy_(0, wide[n:n + m], narrow[n:n + m])
        if n:
            self.lengths.index_copy_(0, wide[:n], narrow[:n])
        return narrow[n + m:]

    def _ints(self, values):
        return self._device(np.asarray(values, np.int32))

    # ------------------------------------------------------------ sequences

    def add(self, rows=0):
        """A new sequence with pages for `rows` rows, which the caller writes; returns its number."""
        n = self._need(rows)
        seq, = self._room(n, 1)
        pages = self._spare(n)
        self._write(self._stage_rows([seq], [pages], [rows]), clear=True)
        self._take(n)
        self._pages[seq], self._len[seq] = pages, rows
        return seq

    def fork(self, seq):
        """A new sequence that shares the pages of `seq`; returns its number."""
        pages = self._held(seq)
        new, = self._room(0, 1)
        self.page_table[new].copy_(self.page_table[seq])
        self.lengths[new].copy_(self.lengths[seq])
        self._refs[pages] += 1
        self._shared += len(pages)
        self._pages[new], self._len[new] = list(pages), self._len[seq]
        return new

    def extend(self, seqs, rows=1):
        """Room for `rows` more rows behind each of `seqs` (distinct), in pages of their own; the caller writes
        them.  Returns the first new row of each (int32, on the device)."""
        if rows < 0 or len(set(seqs)) != len(seqs):
            raise ValueError("rows >= 0 and distinct sequences expected")
        held = [self._held(s) for s in seqs]
        used = self._len[list(seqs)]
        total = used + rows
        if len(seqs):
            self._need(total.max())
        grow = -(-total // self.page_tokens) + -used // self.page_tokens
        copied, left = [], {}
        if rows and self._shared:
            for i in np.flatnonzero(used % self.page_tokens):
                last = held[i][-1]
                # of the sequences that share it, all but the last holder need a copy
                left.setdefault(last, self._refs[last])
                if left[last] > 1:
                    left[last] -= 1
                    copied.append(i)
        wanted = int(grow.sum()) + len(copied)
        self._room(wanted)
        spare = iter(self._spare(wanted))
        own = [(i, next(spare)) for i in copied]                   # in the place of a shared last page
        new = [(i, [next(spare) for _ in range(grow[i])]) for i in np.flatnonzero(grow)]
        entries = [(seqs[i] * self.max_pages + len(held[i]) - 1, p) for i, p in own]
        entries += [(seqs[i] * self.max_pages + len(held[i]) + j, p) for i, pages in new for j, p in enumerate(pages)]
        staged = self._stage(np.asarray(seqs, np.int64), total, entries, used)
        if own:
            apack_copy_pages(self.cache, self._ints([(held[i][-1], p) for i, p in own]))
        first = self._write(staged)
        self._take(wanted)
        for i, p in own:
            self._drop(held[i][-1:])
            held[i][-1] = p
        for i, pages in new:
            held[i] += pages
        self._len[list(seqs)] = total
        return first

    def free(self, seq):
        """Gives up a sequence; pages that no other one shares become free."""
        pages = self._held(seq)
        self.lengths[seq].fill_(0)
        self.page_table[seq].fill_(-1)
        self._drop(pages)
        self._pages[seq], self._len[seq] = None, 0

    # ------------------------------------------------------------ pruning

    def _cache_of(self, lists):
        table = np.full((len(lists), max(1, max(map(len, lists)))), -1, np.int32)
        for i, pages in enumerate(lists):
            table[i, :len(pages)] = pages
        return PagedCache(self.k, self.v, self._ints(table))

    def _split(self, need):
        """Free pages in lists of these lengths (they stay free)."""
        spare = iter(self._spare(sum(need)))
        return [[next(spare) for _ in range(n)] for n in need]

    def prune(self, seqs, keep_idx, kept, in_place=None, ws=None):
        """Keeps kept[i] rows of seqs[i] (distinct): keep_idx holds them, packed over the sequences in this order
        as apack_select writes it (row r of seqs[i] is the sum of the lengths before it + r), ascending.  The kept rows
        go to new pages and the old ones are given up, or, in place, to the first of the sequences' own pages (no
        page of which may be shared) and only the pages behind them are given up: slower (266 against 173 us for a
        two-minute prompt's 24 layers in 16-token pages), but no page is needed.  in_place None: in place only where there are too few
        free pages for the other way."""
        if not len(seqs) or len(set(seqs)) != len(seqs) or len(kept) != len(seqs):
            raise ValueError("distinct sequences and a number of kept rows for each expected")
        lists = [self._held(s) for s in seqs]
        lens = [int(self._len[s]) for s in seqs]
        if any(not 0 <= int(m) <= n for m, n in zip(kept, lens)):
            raise ValueError("kept rows: 0 to the sequence's length")
        need = [self._need(m) for m in kept]
        cu_src, cu_dst = (self._ints(np.concatenate([[0], np.cumsum(x)])) for x in (lens, kept))
        n_out = int(sum(int(m) for m in kept))
        src = self._cache_of(lists)
        own = all(self._refs[p] == 1 for pages in lists for p in pages)
        if in_place and not own:
            raise ValueError("in place: a page is shared with another sequence")
        if in_place is None:
            in_place = own and sum(need) > len(self._free)
        if in_place:
            new = [pages[:n] for n, pages in zip(need, lists)]
            dst = src
        else:
            self._room(sum(need))
            new = self._split(need)
            dst = self._cache_of(new)
        staged = self._stage_rows(seqs, new, kept)
        apack_paged_compact(src, dst, cu_dst, n_out, keep_idx=keep_idx, cu_src=cu_src, ws=ws)
        self._write(staged, clear=True)
        if not in_place:
            self._take(sum(need))
        for s, m, n, pages, now in zip(seqs, kept, need, lists, new):
            self._drop(pages[n:] if in_place else pages)
            self._pages[s], self._len[s] = now, int(m)

    def take(self, src, kept, keep_idx=None, cu_src=None, src_layer=0, dst_layer=0, num_layers=None, ws=None):
        """New sequences from the kept rows of another PagedCache (a prefill's contiguous caches, say: one page of
        all tokens), kept[i] rows of its sequence i; the arguments as in apack_paged_compact.  Returns their numbers.
        Layers of the pool outside dst_layer .. dst_layer + num_layers - 1 hold what the pages held before: the caller
        writes them (apack_paged_compact from their source, into a PagedCache of the pool and the new sequences' pages)
        before they are read."""
        if len(kept) != src.num_seqs:
            raise ValueError(f"kept: {src.num_seqs} numbers expected")
        need = [self._need(m) for m in kept]
        rows = self._room(sum(need), len(kept))
        cu_dst = self._ints(np.concatenate([[0], np.cumsum(kept)]))
        new = self._split(need)
        staged = self._stage_rows(rows, new, kept)
        apack_paged_compact(src, self._cache_of(new), cu_dst, int(sum(int(m) for m in kept)), keep_idx=keep_idx, cu_src=cu_src,
                            src_layer=src_layer, dst_layer=dst_layer, num_layers=num_layers, ws=ws)
        self._write(staged, clear=True)
        self._take(sum(need))
        for s, pages, m in zip(rows, new, kept):
            self._pages[s], self._len[s] = pages, int(m)
        return rows
