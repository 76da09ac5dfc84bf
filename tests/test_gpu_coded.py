"""The cache in 8 bits on the GPU: codes and exponents equal the append rule's, attention is within its roundings of 64 bits."""
import math
import random

import pytest
import torch

import coded_ref as cr
from paged_ref import causal_mask, check, slots, tree_mask

pytestmark = pytest.mark.gpu
DTS = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def rs():
    from paper_2511_01282_gb300 import respec
    return respec


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """Pages in random order; codes and exponents on the GPU (any bytes where nothing was appended)."""

    def __init__(self, lens, page, Hkv, D, seed=0, spare=2):
        g = random.Random(seed)
        need = [-(-x // page) for x in lens]
        self.page, self.Hkv, self.D, self.n = page, Hkv, D, sum(need) + spare
        order = list(range(self.n))
        g.shuffle(order)
        self.most = max(max(need), 1)
        rows, at = [], 0
        for x in need:
            rows.append(order[at:at + x] + [-7] * (self.most - x))
            at += x
        self.table = i32(rows).view(len(lens), self.most)
        gen = torch.Generator().manual_seed(seed)
        byte = lambda *s: torch.randint(0, 256, s, dtype=torch.uint8, generator=gen).cuda()  # noqa: E731
        self.k, self.v = byte(self.n, page, Hkv, D), byte(self.n, page, Hkv, D)
        self.ke, self.ve = (byte(self.n, page // 16, Hkv).view(torch.int8) for _ in range(2))

    def arrays(self):
        return self.k, self.v, self.ke, self.ve

    def args(self, ctx):
        return (*self.arrays(), self.n, self.page, self.table, self.most, ctx)

    def host(self):
        return [x.cpu().clone() for x in self.arrays()]


def append(rs, pool, k, v, off, ctx, T=None):
    status = i32([-1] * len(ctx))
    rs.rs_coded_append(k, k.stride(0), v, v.stride(0), rs.RS_BF16 if k.dtype == torch.bfloat16 else rs.RS_F16, i32(off), len(ctx),
                       k.shape[0] if T is None else T, pool.Hkv, pool.D, *pool.args(i32(ctx)), status)
    return status.tolist()


def attend(rs, pool, q, off, ctx, max_new, scale, parents=None, ws=None, out=None, stream=None):
    B, (T, Hq, D) = len(ctx), q.shape
    out = torch.full((T, Hq, D), 7.0, dtype=q.dtype, device="cuda") if out is None else out
    lse, status = torch.full((T, Hq), 7.0, device="cuda"), i32([-1] * B)
    need = rs.rs_coded_attn_workspace_size(B, T, max_new, Hq, pool.Hkv, D)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
    rs.rs_coded_attn(q, q.stride(0), rs.RS_BF16 if q.dtype == torch.bfloat16 else rs.RS_F16, i32(off), parents, B, T, max_new, Hq,
                     pool.Hkv, D, *pool.args(i32(ctx)), scale, out, lse, status, ws, stream=stream)
    return out, lse, status


def rows(n, heads, D, dt, seed, loud=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, D, generator=g) * torch.exp(loud * torch.randn(n, heads, 1, generator=g))
    return x.to(dt).cuda()


def fill(rs, pool, lens, dt, seed, loud=0.5):
    """Keys and values of every request's first tokens into the pool, some channels louder."""
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    k, v = rows(off[-1], pool.Hkv, pool.D, dt, seed), rows(off[-1], pool.Hkv, pool.D, dt, seed + 1, loud)
    k *= torch.exp(torch.randn(pool.D, generator=torch.Generator().manual_seed(seed + 2))).to(dt).cuda()
    assert append(rs, pool, k, v, off, [0] * len(lens)) == [0] * len(lens)


def check_attention(pool, q, off, ctx, scale, got, parents=None, skip=()):
    out, lse, status = got
    dev = q.device
    k, v = (cr.values(c, e).to(dev).view(-1, pool.Hkv, pool.D) for c, e in ((pool.k, pool.ke), (pool.v, pool.ve)))
    ve = pool.ve.repeat_interleave(16, 1).view(-1, pool.Hkv)
    for b in range(len(ctx)):
        n = off[b + 1] - off[b]
        if b in skip or n == 0:
            continue
        at = slots(pool.table, b, ctx[b] + n, pool.page)
        see = causal_mask(n, ctx[b])
        if parents is not None:
            see = torch.cat([torch.ones(n, ctx[b], dtype=torch.bool), tree_mask(parents[off[b]:off[b + 1]].tolist())], 1)
        want, z, out_tol, lse_tol = cr.coded_attention(q[off[b]:off[b + 1]], k[at], v[at], ve[at], see, scale)
        check(out[off[b]:off[b + 1]], want, out_tol, "out of request %d" % b)
        check(lse[off[b]:off[b + 1]], z, lse_tol, "lse of request %d" % b)
    assert [s for b, s in enumerate(status.tolist()) if b not in skip] == [0] * (len(ctx) - len(skip))


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("Hkv,D,page", [(1, 64, 16), (3, 128, 32), (8, 128, 64), (2, 64, 256)])
def test_append_gives_the_rules_codes(rs, dt, Hkv, D, page):
    lens = [0, 1, 15, 16, 17, 40, 3, 130, 0]
    ctx = [5, 0, 1, 15, 16, 9, 47, 30, 0]
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    pool = Pool([n + c for n, c in zip(lens, ctx)], page, Hkv, D)
    ke, ve = (torch.randint(-9, -4, pool.ke.shape, dtype=torch.int8) for _ in range(2))
    pool.ke, pool.ve = ke.cuda(), ve.cuda()
    k, v = rows(off[-1] + 4, Hkv, D, dt, 1), rows(off[-1] + 4, Hkv, D, dt, 2, 3.0)  # 4 rows behind the last request
    v[7, 0, 3], v[8, 0, 5], v[9, -1, 0], k[20, 0, 1] = math.nan, math.inf, -math.inf, torch.finfo(dt).max
    v[33:33 + 16] = 0.0
    k[40] = torch.finfo(dt).tiny / 4
    want = pool.host()
    for c, e, x in ((want[0], want[2], k), (want[1], want[3], v)):
        cr.append(c, e, pool.table.tolist(), x.cpu(), off, ctx, page)
    assert append(rs, pool, k, v, off, ctx) == [0] * len(ctx)
    for name, a, b in zip(("k", "v", "ke", "ve"), pool.host(), want):
        assert torch.equal(a, b), (name, (a != b).nonzero()[:5], a[a != b][:5], b[a != b][:5])


def test_append_a_token_at_a_time_shifts_what_is_there(rs):
    page, Hkv, D = 16, 2, 64
    pool = Pool([40, 40], page, Hkv, D)
    want = pool.host()
    for i in range(40):
        k, v = rows(2, Hkv, D, torch.bfloat16, 100 + i, 1.5), rows(2, Hkv, D, torch.bfloat16, 200 + i, 1.5)
        assert append(rs, pool, k, v, [0, 1, 2], [i, i]) == [0, 0]
        for c, e, x in ((want[0], want[2], k), (want[1], want[3], v)):
            cr.append(c, e, pool.table.tolist(), x.cpu(), [0, 1, 2], [i, i], page)
    for a, b in zip(pool.host(), want):
        assert torch.equal(a, b)


def test_append_of_parts_of_wider_rows(rs):
    pool, other = Pool([50], 16, 2, 128, 3), Pool([50], 16, 2, 128, 3)
    qkv = rows(50, 8, 128, torch.float16, 4)
    assert append(rs, pool, qkv[:, 4:6], qkv[:, 6:], [0, 50], [0]) == [0]
    assert append(rs, other, qkv[:, 4:6].contiguous(), qkv[:, 6:].contiguous(), [0, 50], [0]) == [0]
    assert all(torch.equal(a, b) for a, b in zip(pool.host(), other.host()))


def test_append_rejects_what_does_not_fit(rs):
    pool = Pool([32, 32], 16, 1, 64)
    k = rows(40, 1, 64, torch.bfloat16, 5)
    before = pool.host()
    for off, ctx in (([0, 33, 40], [0, 33]), ([3, 1, 2], [0, 0]), ([0, 1, 41], [0, 0]), ([-1, 1, 2], [0, 0]), ([0, 1, 2], [-1, 1 << 30])):
        st = append(rs, pool, k, k, off, ctx)
        assert all(s in (0, rs.RS_ST_BAD_OFFSET) for s in st) and rs.RS_ST_BAD_OFFSET in st
    assert append(rs, pool, k, k, [0, 33, 34], [0, 32]) == [rs.RS_ST_BAD_OFFSET] * 2
    assert all(torch.equal(a, b) for a, b in zip(pool.host(), before))
    pool.table[1, 1] = pool.n
    assert append(rs, pool, k, k, [0, 0, 32], [0, 0]) == [0, rs.RS_ST_BAD_PAGE]
    pool.table[1, 1] = -1
    assert append(rs, pool, k, k, [0, 0, 32], [0, 0]) == [0, rs.RS_ST_BAD_PAGE]
    now = pool.host()
    own = int(pool.table[1, 0])
    for a, b in zip(now, before):  # the good page was written, nothing else
        keep = torch.arange(pool.n) != own
        assert torch.equal(a[keep], b[keep]) and not torch.equal(a[own], b[own])


# ------------------------------------------------------------------ attention
SHAPES = [(4, 4, 64, 16), (8, 2, 128, 32), (32, 8, 128, 64), (7, 1, 64, 128), (24, 3, 128, 16), (16, 1, 128, 32), (32, 1, 64, 64), (20, 1, 128, 16)]


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("Hq,Hkv,D,page", SHAPES)
def test_single_tokens(rs, dt, Hq, Hkv, D, page):
    ctx = [0, 1, 15, 16, 17, 255, 1000, 3, 2047]
    off = [0, 1, 2, 3, 4, 5, 6, 7, 7, 8]  # the last but one has none
    pool = Pool([c + 1 for c in ctx], page, Hkv, D)
    fill(rs, pool, [c + 1 for c in ctx], dt, 11)
    q = rows(9, Hq, D, dt, 13)  # and a row behind the last request
    got = attend(rs, pool, q, off, ctx, 1, D ** -0.5)
    check_attention(pool, q, off, ctx, D ** -0.5, got)
    assert (got[0][8] == 7).all() and (got[1][8] == 7).all()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("Hq,Hkv,D,page,n", [(4, 4, 64, 16, 5), (4, 4, 128, 32, 8), (8, 2, 128, 64, 3), (8, 2, 64, 16, 8), (2, 2, 128, 16, 32), (2, 2, 128, 16, 31)])
@pytest.mark.parametrize("tree", [False, True])
def test_a_few_rows(rs, dt, Hq, Hkv, D, page, n, tree):
    ctx, ns = [0, 7, 16, 333, 1201], [n, 1, max(n - 1, 1), 0, n]
    check_rows(rs, dt, Hq, Hkv, D, page, ctx, ns, n, tree)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("Hq,Hkv,D,page,n", [(4, 4, 64, 16, 65), (4, 2, 128, 32, 200), (8, 1, 128, 64, 50), (8, 2, 64, 256, 129), (3, 1, 128, 16, 256)])
@pytest.mark.parametrize("tree", [False, True])
def test_many_rows(rs, dt, Hq, Hkv, D, page, n, tree):
    ctx, ns = [0, 100, 129, 500, 2100], [n, 1, n // 2, 0, n]
    check_rows(rs, dt, Hq, Hkv, D, page, ctx, ns, n, tree)


def check_rows(rs, dt, Hq, Hkv, D, page, ctx, ns, max_new, tree):
    off = [0]
    for x in ns:
        off.append(off[-1] + x)
    lens = [c + x for c, x in zip(ctx, ns)]
    pool = Pool(lens, page, Hkv, D, 5)
    fill(rs, pool, lens, dt, 21)
    q = rows(off[-1] + 2, Hq, D, dt, 23)
    g = random.Random(7)
    parents = i32([-1 if i == 0 else g.randrange(i) for x in ns for i in range(x)] + [0, 0]) if tree else None
    got = attend(rs, pool, q, off, ctx, max_new, D ** -0.5, parents)
    check_attention(pool, q, off, ctx, D ** -0.5, got, parents)
    assert (got[0][-2:] == 7).all() and (got[1][-2:] == 7).all()


@pytest.mark.parametrize("n,G,D", [(1, 4, 128), (1, 8, 64), (70, 2, 128), (70, 2, 64)])
def test_a_long_cache_of_one_request_is_split(rs, n, G, D):
    ctx, dt = [40000], torch.bfloat16
    pool = Pool([ctx[0] + n], 128, 2, D)
    fill(rs, pool, [ctx[0] + n], dt, 31)
    q = rows(n, 2 * G, D, dt, 33) * 3
    got = attend(rs, pool, q, [0, n], ctx, n, D ** -0.5)
    check_attention(pool, q, [0, n], ctx, D ** -0.5, got)
    again = attend(rs, pool, q, [0, n], ctx, n, D ** -0.5)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx,ns", [([8000, 3000], [200, 300]), ([3000, 500, 5000], [8, 300, 70])])
def test_whole_row_tiles_behind_half_ones(rs, D, ctx, ns):
    """Many key tiles to a CTA: pairs of row tiles follow ones whose second row tile has no rows."""
    check_rows(rs, torch.bfloat16, 32, 8, D, 32, ctx, ns, max(ns), False)


@pytest.mark.parametrize("n", [1, 40])
def test_many_requests(rs, n):
    g = random.Random(3)
    ctx = [g.randrange(0, 700) for _ in range(300)]
    ns = [g.randrange(0, n + 1) for _ in ctx]
    check_rows(rs, torch.float16, 4, 2, 64, 16, ctx, ns, n, False)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("n", [1, 40])
def test_exponents_far_apart(rs, dt, n):
    """Blocks of values from the smallest to the largest exponents of the type, keys too."""
    lo, hi = cr.RANGE[dt]
    pool = Pool([400], 32, 2, 64, 9)
    fill(rs, pool, [400], dt, 41, 0.0)
    count = pool.ve.numel()
    wide = torch.linspace(max(lo, -60), min(hi, 40), count).round().to(torch.int8)[torch.randperm(count, generator=torch.Generator().manual_seed(1))]
    pool.ve = wide.view(pool.ve.shape).cuda()
    if dt == torch.float16:  # codes of 2^8 at exponent 8 are above fp16
        pool.v &= 0xbf
    pool.ke = (pool.ke.float() * 0 - 9).to(torch.int8)
    q = rows(n, 4, 64, dt, 43)
    got = attend(rs, pool, q, [0, n], [400 - n], n, 0.125)
    check_attention(pool, q, [0, n], [400 - n], 0.125, got)


@pytest.mark.parametrize("n", [1, 40])
def test_queries_of_any_size(rs, n):
    """bf16 queries far above and below 1, keys that bring the scores back."""
    dt = torch.bfloat16
    for up in (60, -60):
        pool = Pool([200], 16, 1, 64, 9)
        fill(rs, pool, [200], dt, 51)
        pool.ke = (pool.ke.int() - up).to(torch.int8)
        q = (rows(n, 2, 64, dt, 53).float() * 2.0 ** up).to(dt)
        got = attend(rs, pool, q, [0, n], [200 - n], n, 0.125)
        check_attention(pool, q, [0, n], [200 - n], 0.125, got)


@pytest.mark.parametrize("n,max_new", [(1, 1), (8, 8), (40, 40)])
def test_nan_behind_the_last_key_does_not_matter_and_before_it_does(rs, n, max_new):
    dt, D = torch.float16, 64
    pool = Pool([90 + n, 90 + n], 32, 1, D, 4)
    fill(rs, pool, [90 + n, 90 + n], dt, 61)
    for b in range(2):
        end = slots(pool.table, b, 32 * -(-(90 + n) // 32), 32)[90 + n:]
        pool.k.view(-1, 1, D)[end] = 0x7f
        pool.v.view(-1, 1, D)[end] = 0xff
    q = rows(2 * n, 2, D, dt, 63)
    got = attend(rs, pool, q, [0, n, 2 * n], [90, 90], max_new, 0.125)
    check_attention(pool, q, [0, n, 2 * n], [90, 90], 0.125, got)
    at = int(slots(pool.table, 1, 4, 32)[3])
    pool.k.view(-1, 1, D)[at, 0, 5] = 0x7f
    out, lse, status = attend(rs, pool, q, [0, n, 2 * n], [90, 90], max_new, 0.125)
    assert torch.equal(out[:n], got[0][:n]) and out[n:].isnan().all() and lse[n:].isnan().all() and status.tolist() == [0, 0]
    fill(rs, pool, [90 + n, 90 + n], dt, 61)
    pool.v.view(-1, 1, D)[at, 0, 5] = 0xff
    out, lse, status = attend(rs, pool, q, [0, n, 2 * n], [90, 90], max_new, 0.125)
    assert torch.equal(out[:n], got[0][:n]) and out[n:, :, 5].isnan().all() and not out[n:, :, 6].isnan().any() and lse.isfinite().all()


@pytest.mark.parametrize("n", [1, 8, 40])
def test_rejected_requests(rs, n):
    dt, D, Hkv = torch.bfloat16, 64, 2
    lens = [100] * 4
    pool = Pool(lens, 16, Hkv, D, 6)
    fill(rs, pool, lens, dt, 71)
    ctx, off = [100 - n] * 4, [i * n for i in range(5)]
    q = rows(4 * n, 4, D, dt, 73)
    whole = attend(rs, pool, q, off, ctx, n, 0.125)
    check_attention(pool, q, off, ctx, 0.125, whole)

    def expect(got, bad, status):
        out, lse, st = got
        assert st.tolist() == [status if b == bad else 0 for b in range(4)]
        for b in range(4):
            a = slice(off[b], off[b + 1])
            if b == bad:
                assert (out[a] == 0).all() and (lse[a] == 0).all()
            else:
                check_attention(pool, q, off, ctx, 0.125, got, skip=[x for x in range(4) if x != b])

    table = pool.table.clone()
    for page in (-1, pool.n, 1 << 30):
        pool.table[1, 2] = page
        expect(attend(rs, pool, q, off, ctx, n, 0.125), 1, rs.RS_ST_BAD_PAGE)
        pool.table.copy_(table)
    for c in (-1, 16 * pool.most - n + 1, 1 << 30):
        got = attend(rs, pool, q, off, [ctx[0], ctx[1], c, ctx[3]], n, 0.125)
        expect(got, 2, rs.RS_ST_BAD_OFFSET)
    if n > 1:
        got = attend(rs, pool, q, off, ctx, n - 1, 0.125)
        assert got[2].tolist() == [rs.RS_ST_TOO_LARGE] * 4 and (got[0] == 0).all()
        parents = i32([-1] + list(range(n - 1))).repeat(4)
        same = attend(rs, pool, q, off, ctx, n, 0.125, parents)
        check_attention(pool, q, off, ctx, 0.125, same, parents)
        for i, p in ((0, 0), (1, 1), (1, -1), (n - 1, n)):
            bad = parents.clone()
            bad[3 * n + i] = p
            expect(attend(rs, pool, q, off, ctx, n, 0.125, bad), 3, rs.RS_ST_BAD_TREE)
    # ranges outside the rows, or before an earlier request's: left as they are
    for offs, bad in (([0, n, 4 * n + 1, 4 * n + 1, 4 * n + 1], (1, 2, 3)), ([n, 2 * n, n, 2 * n, 3 * n], (1, 2))):
        out, lse, st = attend(rs, pool, q, offs, ctx, n, 0.125)
        assert all(st.tolist()[b] == rs.RS_ST_BAD_OFFSET for b in bad)
        check_attention(pool, q, offs, ctx, 0.125, (out, lse, st), skip=bad) if st.tolist()[0] == 0 else None


@pytest.mark.parametrize("n", [1, 40])
def test_no_requests_and_no_rows(rs, n):
    pool = Pool([50, 50], 16, 2, 64)
    q = rows(3, 4, 64, torch.bfloat16, 1)
    out, lse, st = attend(rs, pool, q, [0, 0, 0], [10, 0], n, 0.1)
    assert (out == 7).all() and (lse == 7).all() and st.tolist() == [0, 0]
    assert append(rs, pool, q[:, :2], q[:, 2:], [0, 0, 0], [10, 0]) == [0, 0]
    st = i32([-1, -1])
    ws = torch.empty(rs.rs_coded_attn_workspace_size(2, 0, n, 4, 2, 64), dtype=torch.uint8, device="cuda")
    rs.rs_coded_attn(None, 256, 0, i32([0, 0, 0]), None, 2, 0, n, 4, 2, 64, *pool.args(i32([0, 0])), 0.1, None, None, st, ws)
    assert st.tolist() == [0, 0]


@pytest.mark.parametrize("n", [1, 40])
def test_graphs_and_streams(rs, n):
    dt, D = torch.bfloat16, 128
    ctx, off = [300, 700], [0, n, 2 * n]
    pool = Pool([c + n for c in ctx], 32, 2, D, 8)
    fill(rs, pool, [c + n for c in ctx], dt, 81)
    k, v, q = rows(2 * n, 2, D, dt, 83), rows(2 * n, 2, D, dt, 84), rows(2 * n, 8, D, dt, 85)
    first = pool.host()
    assert append(rs, pool, k, v, off, ctx) == [0, 0]
    want, after = attend(rs, pool, q, off, ctx, n, 0.1), pool.host()
    offs, cs = i32(off), i32(ctx)
    out, lse, st = torch.zeros_like(q), torch.zeros(2 * n, 8, device="cuda"), i32([-1, -1])
    ws = torch.empty(rs.rs_coded_attn_workspace_size(2, 2 * n, n, 8, 2, D), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        rs.rs_coded_append(k, 2 * D, v, 2 * D, rs.RS_BF16, offs, 2, 2 * n, 2, D, *pool.args(cs), st, stream=stream)
        rs.rs_coded_attn(q, 8 * D, rs.RS_BF16, offs, None, 2, 2 * n, n, 8, 2, D, *pool.args(cs), 0.1, out, lse, st, ws, stream=stream)

    side = torch.cuda.Stream()
    for how in ("stream", "graph", "graph"):
        for x, y in zip(pool.arrays(), first):
            x.copy_(y)
        out.zero_()
        torch.cuda.synchronize()
        if how == "stream":
            step(side)
        else:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
            eager = attend(rs, pool, q, off, ctx, n, 0.1)  # beside it, with a workspace of its own
            graph.replay()
            assert torch.equal(eager[0], want[0])
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and st.tolist() == [0, 0]
        assert all(torch.equal(a, b) for a, b in zip(pool.host(), after))


@pytest.mark.parametrize("n", [1, 40])
def test_offsets_past_32_bits(rs, n):
    """A pool of more than 2^32 bytes: the last pages' codes are found."""
    D, Hkv, page = 128, 8, 4096
    pages = (1 << 32) // (page * Hkv * D) + 3
    pool = Pool([n + 300], page, Hkv, D, 2, spare=0)
    small = pool.host()
    pool.n = pages
    pool.k, pool.v = (torch.zeros(pages, page, Hkv, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    pool.ke, pool.ve = (torch.zeros(pages, page // 16, Hkv, dtype=torch.int8, device="cuda") for _ in range(2))
    pool.table[:] = pages - 1
    fill(rs, pool, [n + 300], torch.bfloat16, 91)
    assert pool.k[-1].any() and not pool.k[:-1].any() and len(small) == 4
    q = rows(n, 16, D, torch.bfloat16, 93)
    got = attend(rs, pool, q, [0, n], [300], n, 0.1)
    last = Pool([n + 300], page, Hkv, D, 2, spare=0)
    last.table[:] = 0
    last.n = 1
    last.k, last.v, last.ke, last.ve = (x[-1:].clone() for x in pool.arrays())
    check_attention(last, q, [0, n], [300], 0.1, got)
