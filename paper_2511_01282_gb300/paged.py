"""A paged KV cache of one attention layer: device buffers plus the paged calls in order.

``PagedCache`` holds the pages, the page table and, where eviction is wanted, every key's accumulated weight and position.
A program appends the new tokens' keys and values, attends with their queries, and then says how many of them stay
(``advance``); what was appended behind them is written over by the next ``append``.  ``prompt_attention`` is the pass over
whole prompts that comes before.
"""
import torch

from . import respec as rs

_CODES = {torch.bfloat16: rs.RS_BF16, torch.float16: rs.RS_F16}


def _scratch(held, need, device):
    """A buffer of at least `need` bytes: the one held where it is large enough."""
    if held is None or held.numel() < need:
        held = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return held


def prompt_attention(q, k, v, seq_off, scale, workspace=None):
    """Causal attention of packed prompts (rs_prompt_attn): q [T, Hq, D], k and v [T, Hkv, D] (rows may be parts of wider
    ones), seq_off [B+1] int32 on the device.  Returns (out, lse, status, workspace)."""
    T, Hq, D = q.shape
    Hkv, B, dev = k.shape[1], seq_off.numel() - 1, q.device
    out = torch.empty((T, Hq, D), dtype=q.dtype, device=dev)
    lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    workspace = _scratch(workspace, rs.rs_prompt_attn_workspace_size(B, T, Hq, Hkv, D), dev)
    rs.rs_prompt_attn(q, q.stride(0), k, k.stride(0), v, v.stride(0), _CODES[q.dtype], seq_off, B, T, Hq, Hkv, D, scale, out, lse,
                      status, workspace)
    return out, lse, status, workspace


class PagedCache:
    """B requests with `tokens` slots each, in pages of `page_size` tokens."""

    def __init__(self, B, tokens, page_size, Hkv, D, dtype=torch.bfloat16, track_weights=False, device="cuda"):
        self.B, self.page_size, self.Hkv, self.D, self.dtype = B, page_size, Hkv, D, dtype
        self.max_pages = -(-tokens // page_size)
        self.n_pages = B * self.max_pages
        self.device = torch.device(device)
        z = lambda *s, dt: torch.zeros(s, dtype=dt, device=self.device)  # noqa: E731
        self.k, self.v = z(self.n_pages, page_size, Hkv, D, dt=dtype), z(self.n_pages, page_size, Hkv, D, dt=dtype)
        self.table = torch.arange(self.n_pages, dtype=torch.int32, device=self.device).view(B, self.max_pages)
        self.length = z(B, dt=torch.int32)  # cached tokens
        self.lengths = [0] * B              # the same on the host
        slots = self.n_pages * page_size
        self.weights = z(Hkv, slots, dt=torch.float32) if track_weights else None
        self.positions = z(Hkv, slots, dt=torch.int32) if track_weights else None
        self.status = z(B, dt=torch.int32)
        self._ws = None

    def _pages(self):
        return self.n_pages, self.page_size, self.table, self.max_pages

    def append(self, k, v, new_off, pos=None):
        """Keys and values [T, Hkv, D] of new tokens behind the cached ones; pos [T] their positions."""
        rs.rs_paged_append(k, k.stride(0), v, v.stride(0), pos, new_off, self.B, k.shape[0], self.Hkv, self.D, self.k, self.v,
                           *self._pages(), self.length, self.weights, self.positions, self.status)

    def attend(self, q, new_off, scale, parents=None):
        """Attention of the appended tokens' queries [T, Hq, D]: (out, lse)."""
        T, Hq, D = q.shape
        out = torch.empty((T, Hq, D), dtype=q.dtype, device=self.device)
        lse = torch.empty((T, Hq), dtype=torch.float32, device=self.device)
        self._ws = _scratch(self._ws, rs.rs_paged_attn_workspace_size(self.B, T, Hq, self.Hkv, D), self.device)
        rs.rs_paged_attn(q, q.stride(0), _CODES[q.dtype], new_off, parents, self.B, T, Hq, self.Hkv, D, self.k, self.v, *self._pages(),
                         self.length, scale, out, lse, self.status, self._ws)
        return out, lse

    def weigh(self, q, lse, new_off, scale):
        """Adds the weight that rows q [T, Hq, D] (causal, behind the cached tokens) give to every key they see."""
        T, Hq, D = q.shape
        self._ws = _scratch(self._ws, rs.rs_paged_weights_workspace_size(self.B, T, Hq, self.Hkv, D), self.device)
        rs.rs_paged_weights(q, q.stride(0), _CODES[q.dtype], lse, new_off, self.B, T, Hq, self.Hkv, D, self.k, *self._pages(),
                            self.length, scale, self.weights, self.status, self._ws)

    def rows(self, b, slots):
        """Pool rows of request b's slots (a device index tensor)."""
        return self.table[b].long()[slots // self.page_size] * self.page_size + slots % self.page_size

    def keep(self, b, nodes):
        """Of the tokens appended behind request b's cached ones, `nodes` (ascending) come first: the accepted path of a tree."""
        at = torch.as_tensor(nodes, dtype=torch.int64, device=self.device) + self.lengths[b]
        src, dst = self.rows(b, at), self.rows(b, torch.arange(len(nodes), device=self.device) + self.lengths[b])
        for x in (self.k, self.v):
            x = x.view(-1, self.Hkv, self.D)
            x[dst] = x[src]
        if self.positions is not None:
            self.positions[:, dst] = self.positions[:, src]

    def advance(self, counts):
        """The first counts[b] of the appended tokens stay."""
        self._set([n + c for n, c in zip(self.lengths, counts)])

    def evict(self, next_pos, budget, recent):
        """Cuts every request to `budget` tokens per head; next_pos[b]: tokens that request b has seen."""
        self._ws = _scratch(self._ws, rs.rs_paged_evict_workspace_size(self.B, self.Hkv, budget), self.device)
        new = torch.empty_like(self.length)
        nxt = torch.tensor(next_pos, dtype=torch.int32, device=self.device)
        rs.rs_paged_evict(self.k, self.v, self.Hkv, self.D, *self._pages(), self.length, nxt, self.B, budget, recent, self.weights,
                          self.positions, new, self.status, self._ws)
        self._set([min(n, budget) for n in self.lengths])

    def _set(self, lengths):
        self.lengths = list(lengths)
        self.length.copy_(torch.tensor(self.lengths, dtype=torch.int32))
