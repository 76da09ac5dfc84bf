"""A paged KV cache of one attention layer: device buffers plus the paged calls in order.

``PagedCache`` holds the pages, the page table and, where eviction is wanted, every key's accumulated weight and position.
A program appends the new tokens' keys and values, attends with their queries, and then says how many of them stay
(``advance``); what was appended behind them is written over by the next ``append``.  ``prompt_attention`` is the pass over
whole prompts that comes before.  ``append``, ``attend`` and ``weigh`` may be captured into a CUDA graph; the others copy from
the host.  What the calls report about requests (bad pages, a time-out) is gathered on the device: ``check`` reads it and raises.
"""
import torch

from . import respec as rs

_CODES = {torch.bfloat16: rs.RS_BF16, torch.float16: rs.RS_F16}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _heads(name, x, heads, D, dtype):
    """x is [rows, heads, D] of the type; heads None: any number."""
    _need(x.dim() == 3 and x.shape[2] == D and heads in (None, x.shape[1]) and x.dtype == dtype,
          "%s: [rows, %s, %d] of %s expected, not %s of %s" % (name, heads or "heads", D, dtype, list(x.shape), x.dtype))


def _apart(x):
    """Elements from row to row of [rows, heads, D]; what a tensor has for a single row means nothing."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1] * x.shape[2]


def _ints(name, x, n):
    _need(x.dtype == torch.int32 and x.dim() == 1 and x.numel() == n, "%s: %d values of int32 expected, not %s of %s"
          % (name, n, list(x.shape), x.dtype))


_STATUS = [n for n in dir(rs) if n.startswith("RS_ST_")]


def _flags(status):
    return " ".join(n[6:] for n in _STATUS if status & getattr(rs, n)) or "status %d" % status


def _raise(status):
    raise RuntimeError("; ".join("request %d: %s" % (b, _flags(x)) for b, x in enumerate(status) if x))


def _scratch(need, device):
    return torch.empty(max(need, 256), dtype=torch.uint8, device=device)


def prompt_attention(q, k, v, seq_off, scale, workspace=None):
    """Causal attention of packed prompts (rs_prompt_attn): q [T, Hq, D], k and v [T, Hkv, D] (rows may be parts of wider
    ones), seq_off [B+1] int32 on the device.  Returns (out, lse, status, workspace); a workspace that is handed in again is used
    where it is large enough."""
    _need(q.dtype in _CODES and q.dim() == 3, "q: [rows, heads, D] of bfloat16 or float16 expected")
    T, Hq, D = q.shape
    for name, x in (("k", k), ("v", v)):
        _heads(name, x, k.shape[1] if x is v else None, D, q.dtype)
        _need(x.shape[0] == T, "%s: %d rows expected, not %d" % (name, T, x.shape[0]))
    Hkv, B, dev = k.shape[1], seq_off.numel() - 1, q.device
    _ints("seq_off", seq_off, B + 1)
    out = torch.empty((T, Hq, D), dtype=q.dtype, device=dev)
    lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    need = rs.rs_prompt_attn_workspace_size(B, T, Hq, Hkv, D)
    if workspace is None or workspace.numel() < need:
        workspace = _scratch(need, dev)
    rs.rs_prompt_attn(q, _apart(q), k, _apart(k), v, _apart(v), _CODES[q.dtype], seq_off, B, T, Hq, Hkv, D, scale, out, lse,
                      status, workspace)
    return out, lse, status, workspace


class PagedCache:
    """B requests with `tokens` slots each, in pages of `page_size` tokens.  Every request owns its pages for good: an eviction bounds
    what the calls read, not the memory.  (The library's calls take any page table.)"""

    def __init__(self, B, tokens, page_size, Hkv, D, dtype=torch.bfloat16, track_weights=False, device="cuda"):
        _need(dtype in _CODES and D in (64, 128), "dtype=%s, D=%d: bfloat16 or float16, 64 or 128 expected" % (dtype, D))
        _need(8 <= page_size <= 65536 and page_size & (page_size - 1) == 0, "page_size=%d: a power of two from 8 to 65536 expected" % page_size)
        _need(B >= 0 and tokens >= 0 and Hkv >= 1, "B=%d, tokens=%d, Hkv=%d: out of range" % (B, tokens, Hkv))
        _need(B * -(-tokens // page_size) * page_size < (1 << 31) - 65536, "%d requests of %d tokens: 2^31 slots or more" % (B, tokens))
        self.B, self.page_size, self.Hkv, self.D, self.dtype = B, page_size, Hkv, D, dtype
        self.max_pages = -(-tokens // page_size)
        self.n_pages = B * self.max_pages
        self.device = torch.device(device)
        z = lambda *s, dt: torch.zeros(s, dtype=dt, device=self.device)  # noqa: E731
        self.k, self.v = z(self.n_pages, page_size, Hkv, D, dt=dtype), z(self.n_pages, page_size, Hkv, D, dt=dtype)
        self.table = torch.arange(self.n_pages, dtype=torch.int32, device=self.device).view(B, self.max_pages)
        # cached tokens, and the position of the next one (behind an eviction it is the higher); the same on the host
        self._counts = z(2, B, dt=torch.int32)
        self.length, self.next = self._counts.unbind()
        self.lengths, self.seen = [0] * B, [0] * B
        self._numbered = False  # the last tokens came without positions
        slots = self.n_pages * page_size
        self.weights = z(Hkv, slots, dt=torch.float32) if track_weights else None
        self.positions = z(Hkv, slots, dt=torch.int32) if track_weights else None
        self.status = z(B, dt=torch.int32)  # RS_ST_* flags of all calls since the last check

    def report(self, status):
        """A call's status [B] joins those that `check` looks at (on the device: it may be captured)."""
        self.status |= status

    def check(self):
        """Raises where a call since the last check has reported something about a request; waits for the calls."""
        found = self.status.tolist()
        if any(found):
            self.status.zero_()
            _raise(found)

    def _reported(self, call, *args, workspace=()):
        status = torch.empty_like(self.status)
        call(*args, status, *workspace)
        self.report(status)

    def _pages(self):
        return self.n_pages, self.page_size, self.table, self.max_pages

    def append(self, k, v, new_off, pos=None):
        """Keys and values [T, Hkv, D] of new tokens behind the cached ones; pos [T] their positions (where the cache keeps any):
        without it they go on from the tokens that the request has seen."""
        T = k.shape[0]
        for name, x in (("k", k), ("v", v)):
            _heads(name, x, self.Hkv, self.D, self.dtype)
        _need(v.shape[0] == T, "v: %d rows expected, not %d" % (T, v.shape[0]))
        _ints("new_off", new_off, self.B + 1)
        self._numbered = pos is None
        if pos is not None:
            _ints("pos", pos, T)
        elif self.positions is not None and T > 0 and self.B > 0:
            pos = self._numbers(T, new_off)
        self._reported(rs.rs_paged_append, k, _apart(k), v, _apart(v), pos, new_off, self.B, T, self.Hkv, self.D, self.k, self.v,
                       *self._pages(), self.length, self.weights, self.positions)

    def _numbers(self, T, new_off):
        """Row i of request b: next[b] + i, on the device (the library's own numbers are slots, which fall behind where tokens
        have been evicted)."""
        at = torch.arange(T, dtype=torch.int32, device=self.device)
        b = torch.searchsorted(new_off[1:], at, right=True).clamp_(max=self.B - 1)
        return self.next[b] + at - new_off[b]

    def attend(self, q, new_off, scale, parents=None):
        """Attention of the appended tokens' queries [T, Hq, D]: (out, lse)."""
        _heads("q", q, None, self.D, self.dtype)
        T, Hq, D = q.shape
        _ints("new_off", new_off, self.B + 1)
        if parents is not None:
            _ints("parents", parents, T)
        out = torch.empty((T, Hq, D), dtype=q.dtype, device=self.device)
        lse = torch.empty((T, Hq), dtype=torch.float32, device=self.device)
        ws = _scratch(rs.rs_paged_attn_workspace_size(self.B, T, Hq, self.Hkv, D), self.device)
        self._reported(rs.rs_paged_attn, q, _apart(q), _CODES[q.dtype], new_off, parents, self.B, T, Hq, self.Hkv, D, self.k, self.v,
                       *self._pages(), self.length, scale, out, lse, workspace=(ws,))
        return out, lse

    def weigh(self, q, lse, new_off, scale):
        """Adds the weight that rows q [T, Hq, D] (causal, behind the cached tokens) give to every key they see."""
        _heads("q", q, None, self.D, self.dtype)
        T, Hq, D = q.shape
        _need(lse.shape == (T, Hq) and lse.dtype == torch.float32, "lse: [%d, %d] of float32 expected" % (T, Hq))
        _ints("new_off", new_off, self.B + 1)
        self._tracked()
        ws = _scratch(rs.rs_paged_weights_workspace_size(self.B, T, Hq, self.Hkv, D), self.device)
        self._reported(rs.rs_paged_weights, q, _apart(q), _CODES[q.dtype], lse, new_off, self.B, T, Hq, self.Hkv, D, self.k,
                       *self._pages(), self.length, scale, self.weights, workspace=(ws,))

    def rows(self, b, slots):
        """Pool rows of request b's slots (a device index tensor; slots below the capacity: the lookup does not check)."""
        return self.table[b].long()[slots // self.page_size] * self.page_size + slots % self.page_size

    def keep(self, b, nodes):
        """Of the tokens appended behind request b's cached ones, `nodes` (ascending) come first: the accepted path of a tree.
        Positions that the append was given go with them; without any the path's tokens follow each other."""
        nodes = torch.as_tensor(nodes, dtype=torch.int64).tolist()
        _need(0 <= b < self.B, "request %d: there are %d" % (b, self.B))
        _need(all(0 <= x < self.max_pages * self.page_size - self.lengths[b] for x in nodes),
              "nodes: tokens behind the %d cached ones expected, %d slots in all" % (self.lengths[b], self.max_pages * self.page_size))
        at = torch.tensor(nodes, dtype=torch.int64, device=self.device) + self.lengths[b]
        src, dst = self.rows(b, at), self.rows(b, torch.arange(len(nodes), device=self.device) + self.lengths[b])
        for x in (self.k, self.v):
            x = x.view(-1, self.Hkv, self.D)
            x[dst] = x[src]
        if self.positions is not None:
            if self._numbered:
                self.positions[:, dst] = torch.arange(len(nodes), dtype=torch.int32, device=self.device) + self.seen[b]
            else:
                self.positions[:, dst] = self.positions[:, src]

    def advance(self, counts):
        """The first counts[b] of the appended tokens stay."""
        _need(len(counts) == self.B and all(c >= 0 and n + c <= self.max_pages * self.page_size for n, c in zip(self.lengths, counts)),
              "counts: a number of tokens for each of %d requests, %d cached ones at most" % (self.B, self.max_pages * self.page_size))
        self._set([n + c for n, c in zip(self.lengths, counts)], [n + c for n, c in zip(self.seen, counts)])

    def evict(self, next_pos, budget, recent):
        """Cuts every request to `budget` tokens per head; next_pos[b]: tokens that request b has seen (later ones are counted
        on from there).  A request that the call rejects keeps its tokens, and this raises."""
        _need(len(next_pos) == self.B, "next_pos: a position for each of %d requests" % self.B)
        self._tracked()
        ws = _scratch(rs.rs_paged_evict_workspace_size(self.B, self.Hkv, budget), self.device)
        both = torch.empty((2, self.B), dtype=torch.int32, device=self.device)
        new, status = both.unbind()
        seen = [int(x) for x in next_pos]
        nxt = torch.tensor(seen, dtype=torch.int32, device=self.device)
        rs.rs_paged_evict(self.k, self.v, self.Hkv, self.D, *self._pages(), self.length, nxt, self.B, budget, recent, self.weights,
                          self.positions, new, status, ws)
        torch.stack((new, nxt), out=self._counts)
        (self.lengths, found), self.seen = both.tolist(), seen
        if any(found):
            _raise(found)

    def _tracked(self):
        _need(self.weights is not None, "a cache made with track_weights=True expected")

    def _set(self, lengths, seen):
        self.lengths, self.seen = list(lengths), list(seen)
        self._counts.copy_(torch.tensor([self.lengths, self.seen], dtype=torch.int32))
