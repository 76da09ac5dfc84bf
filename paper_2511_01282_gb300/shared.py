"""A paged KV cache whose requests take their pages from one pool and share those that they have in common.

``reserve`` gives requests the pages for the tokens to come, ``fork`` lets a request go on from another's tokens (a common prompt,
branches of one answer), ``free`` and ``trim`` give pages back, ``resize`` closes the pool up and makes it smaller or larger.  Which
pages are used is kept on the host; the arrays are moved on the device (``rs_pages_copy``, ``rs_pages_compact``).  None of the five
may be captured into a CUDA graph, and graphs of the other calls hold on to the arrays that ``resize`` replaces.
"""
from itertools import islice

import torch

from . import respec as rs
from .paged import PagedCache, _need, _scratch


class SharedCache(PagedCache):
    """B places for requests of `tokens` tokens at most (rounded up to whole pages), over a pool of `pages` pages of `page_size`; a place holds no page at first.

    Whole pages of a common prefix are shared, and nothing writes to them: new tokens come behind them.  With track_weights every
    request has pages of its own (weights are a request's, and an eviction moves tokens within its pages): fork copies them."""

    def __init__(self, B, tokens, page_size, Hkv, D, pages, dtype=torch.bfloat16, track_weights=False, device="cuda", bits=16):
        _need(pages >= 0, "pages=%d: out of range" % pages)
        self._size = pages
        super().__init__(B, tokens, page_size, Hkv, D, dtype, track_weights, device, bits)
        self.held = [[] for _ in range(B)]  # each request's pages, in order
        self.refs = [0] * pages
        self._free = list(range(pages - 1, -1, -1))

    def _pool_pages(self):
        return self._size

    def _first_table(self):
        return torch.full((self.B, self.max_pages), -1, dtype=torch.int32, device=self.device)

    def slots(self, b):
        return len(self.held[b]) * self.page_size

    @property
    def free_pages(self):
        return len(self._free)

    def _place(self, b):
        _need(0 <= b < self.B, "request %d: there are %d" % (b, self.B))

    def _take(self, pages):
        """pages: the first that _spare has given."""
        del self._free[len(self._free) - len(pages):]
        for p in pages:
            self.refs[p] = 1

    def _spare(self):
        """The free pages in the order in which they are given out."""
        return reversed(self._free)

    def _give(self, pages):
        for p in pages:
            self.refs[p] -= 1
            if self.refs[p] == 0:
                self._free.append(p)

    # A call makes ready on the device all that it needs before it changes anything: one that fails leaves the cache as it was.
    def _entries(self, changes):
        """changes: (request, first entry, pages) of the table, as _enter takes them; in one copy."""
        at = [b * self.max_pages + first + i for b, first, pages in changes for i in range(len(pages))]
        if not at:
            return None
        both = torch.tensor([at, [p for _, _, pages in changes for p in pages]], dtype=torch.int64).to(self.device)
        return both[0], both[1].int()

    def _enter(self, entries):
        if entries:
            at, pages = entries
            self.table.view(-1)[at] = pages

    def reserve(self, counts):
        """Pages for counts[b] tokens behind request b's cached ones.  Raises, and takes none, where the pool has too few."""
        _need(len(counts) == self.B and all(c >= 0 and n + c <= self.max_pages * self.page_size for n, c in zip(self.lengths, counts)),
              "counts: a number of tokens for each of %d requests, %d cached ones at most" % (self.B, self.max_pages * self.page_size))
        more = [max(0, -(-(n + c) // self.page_size) - len(h)) if c else 0 for n, c, h in zip(self.lengths, counts, self.held)]
        if sum(more) > len(self._free):
            raise MemoryError("%d pages needed, %d of %d free" % (sum(more), len(self._free), self.n_pages))
        spare = self._spare()
        changes = [(b, len(self.held[b]), list(islice(spare, n))) for b, n in enumerate(more) if n]
        self._enter(self._entries(changes))
        for b, _, own in changes:
            self._take(own)
            self.held[b] += own

    def fork(self, src, dsts, n=None):
        """Requests dsts, which hold nothing, go on from the first n of request src's cached tokens (None: all of them)."""
        dsts = list(dsts)
        for b in [src] + dsts:
            self._place(b)
        _need(len(set(dsts)) == len(dsts) and not any(self.held[b] for b in dsts), "dsts: different requests without pages expected")
        n = self.lengths[src] if n is None else n
        _need(0 <= n <= self.lengths[src], "n=%d: request %d has %d tokens" % (n, src, self.lengths[src]))
        # an evicted request's tokens are in no order, so there is no first part of them
        _need(self.weights is None or n == self.lengths[src], "n=%d: all %d tokens expected where weights are kept" % (n, self.lengths[src]))
        used = -(-n // self.page_size)
        whole = 0 if self.weights is not None else n // self.page_size
        if len(dsts) * (used - whole) > len(self._free):
            raise MemoryError("%d pages needed, %d of %d free" % (len(dsts) * (used - whole), len(self._free), self.n_pages))
        spare = self._spare()
        own = [list(islice(spare, used - whole)) for _ in dsts]
        held = [self.held[src][:whole] + o for o in own]
        pairs = [pr for o in own for pr in zip(self.held[src][whole:used], o)]
        entries = self._entries([(b, 0, h) for b, h in zip(dsts, held)])
        if pairs:
            status = torch.empty(1, dtype=torch.int32, device=self.device)
            rs.rs_pages_copy(*self._moved(), torch.tensor(pairs, dtype=torch.int32, device=self.device), len(pairs), status)
            self.report(status)
        lengths, seen = list(self.lengths), list(self.seen)
        for b in dsts:
            lengths[b], seen[b] = n, seen[src] - lengths[src] + n
        self._set(lengths, seen)
        self._enter(entries)
        for b, h, o in zip(dsts, held, own):
            self._take(o)
            for p in h[:whole]:
                self.refs[p] += 1
            self.held[b] = h

    def _moved(self):
        return (*self._arrays(), self.weights, self.positions, self.bits, self.Hkv, self.D, self.n_pages, self.page_size)

    def _cut(self, b, pages, counts=None):
        gone = self.held[b][pages:]
        entries = self._entries([(b, pages, [-1] * len(gone))])
        if counts is not None:
            self._set(*counts)
        self._enter(entries)
        self.held[b] = self.held[b][:pages]
        self._give(gone)

    def trim(self, b):
        """Request b's pages behind its cached tokens go back to the pool."""
        self._place(b)
        self._cut(b, -(-self.lengths[b] // self.page_size))

    def free(self, b):
        """Request b ends: its place holds nothing."""
        self._place(b)
        lengths, seen = list(self.lengths), list(self.seen)
        lengths[b] = seen[b] = 0
        self._cut(b, 0, (lengths, seen))

    def compact(self):
        """The used pages come to lie in front, one behind the other.  Returns their number; waits for the device (a pool of 16384 pages
        with a quarter in use: 2 ms, most of it for the host's lists of pages)."""
        held, refs = (torch.tensor(x, dtype=torch.int32, device=self.device) for x in ([len(h) for h in self.held], self.refs))
        both = torch.empty(self.n_pages + self.B, dtype=torch.int32, device=self.device)
        new_id, status = both[:self.n_pages], both[self.n_pages:]
        ws = _scratch(rs.rs_pages_compact_workspace_size(self.n_pages), self.device)
        rs.rs_pages_compact(*self._moved(), self.table, self.max_pages, held, self.B, refs, new_id, status, ws)
        self.report(status)
        moved = both[:self.n_pages].tolist()
        used = self.n_pages - len(self._free)
        refs = [0] * self.n_pages
        for p, r in enumerate(self.refs):
            if r:
                refs[moved[p]] = r
        self.refs = refs
        self.held = [[moved[p] for p in h] for h in self.held]
        self._free = list(range(self.n_pages - 1, used - 1, -1))
        return used

    def resize(self, pages):
        """The pool with `pages` pages instead: its used ones are moved to the front first.  Both pools are held until all is copied."""
        used = self.n_pages - len(self._free)
        _need(pages >= used, "pages=%d: %d are used" % (pages, used))
        _need(pages * self.page_size < (1 << 31) - 65536, "pages=%d: 2^31 slots or more" % pages)
        self.compact()

        def sized(x, dim, n, used):
            if x is None:
                return None
            shape = list(x.shape)
            shape[dim] = n
            out = torch.zeros(shape, dtype=x.dtype, device=x.device)
            out.narrow(dim, 0, used).copy_(x.narrow(dim, 0, used))
            return out

        slots = self.page_size
        arrays = [sized(x, 0, pages, used) for x in self._arrays()]
        arrays += [sized(x, 1, pages * slots, used * slots) for x in (self.weights, self.positions)]
        self.k, self.v, self.k_exps, self.v_exps, self.weights, self.positions = arrays
        self.n_pages = self._size = pages
        self.refs = self.refs[:used] + [0] * (pages - used)
        self._free = list(range(pages - 1, used - 1, -1))
