"""Attention over the cache in 8 bits where single calls of ordinary sizes do not go: caches so long that KV heads are read side by
side, waits that run out, two calls at once, sizes that reject one of many requests."""
import math
import random

import pytest
import torch

import coded_ref as cr
from paged_ref import causal_mask, slots, tree_mask
from test_gpu_coded import Pool, append, attend, check_attention, fill, i32, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs():
    from paper_2511_01282_gb300 import respec
    return respec


# The few-row kernel takes several KV heads of a block side by side from 64 blocks and heads a CTA on: with 152 SMs of three
# CTAs (two from nine rows on), 29184 (19456) of them, so with 4 heads 117000 tokens, with 2 at a time of 6 heads 78000.
@pytest.mark.parametrize("Hq,Hkv,D,page,n,tree,dt", [
    (16, 4, 64, 64, 1, False, torch.float16), (12, 6, 64, 16, 3, False, torch.bfloat16), (8, 4, 128, 128, 4, True, torch.bfloat16),
    (16, 8, 64, 32, 8, True, torch.float16), (12, 6, 128, 256, 16, False, torch.bfloat16)])
def test_long_caches_with_heads_side_by_side(rs, Hq, Hkv, D, page, n, tree, dt):
    rows_ = n * Hq // Hkv
    need = 64 * (456 if rows_ <= 8 else 304) // Hkv * 16
    ctx = [0, need // 2, 5, 31, need // 4 + 3, 1000, need // 4 + 900, 0]
    ns = [n, n, 1, 0, max(n - 1, 1), n, n, 1]
    off = [0]
    for x in ns:
        off.append(off[-1] + x)
    lens = [c + x for c, x in zip(ctx, ns)]
    assert sum(-(-x // 16) for x, k in zip(lens, ns) if k) * Hkv >= 64 * (456 if rows_ <= 8 else 304)
    pool = Pool(lens, page, Hkv, D, 5)
    fill(rs, pool, lens, dt, 21)
    q = rows(off[-1] + 2, Hq, D, dt, 23)
    g = random.Random(7)
    parents = i32([-1 if i == 0 else g.randrange(i) for x in ns for i in range(x)] + [0, 0]) if tree else None
    got = attend(rs, pool, q, off, ctx, n, D ** -0.5, parents)
    check_attention(pool, q, off, ctx, D ** -0.5, got, parents)
    assert (got[0][-2:] == 7).all() and (got[1][-2:] == 7).all()
    again = attend(rs, pool, q, off, ctx, n, D ** -0.5, parents)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # a bad page in the middle of a long request: that one is emptied, the others keep their bits
    pool.table[4, (need // 8) // page] = pool.n
    bad = attend(rs, pool, q, off, ctx, n, D ** -0.5, parents)
    assert bad[2].tolist() == [rs.RS_ST_BAD_PAGE if b == 4 else 0 for b in range(8)]
    a, e = off[4], off[5]
    assert (bad[0][a:e] == 0).all() and (bad[1][a:e] == 0).all()
    for x, y in zip(bad[:2], got[:2]):
        assert torch.equal(x[:a], y[:a]) and torch.equal(x[e:], y[e:])


@pytest.mark.parametrize("n", [1, 300])
def test_waits_that_run_out_report_it(rs, n, monkeypatch):
    """A limit of one cycle: the pipelines give up, say so, and the next call works.  (A try to pass a barrier itself waits for some
    microseconds, so there is enough to do for one to fail.)"""
    dt, D, Hkv, B = torch.bfloat16, 128, 8, 8
    lens = [20000 + n] * B
    pool = Pool(lens, 64, Hkv, D, 6)
    fill(rs, pool, lens, dt, 71)
    ctx, off = [20000] * B, [i * n for i in range(B + 1)]
    q = rows(B * n, 32, D, dt, 73)
    want = attend(rs, pool, q, off, ctx, n, 0.09)
    assert want[2].tolist() == [0] * B
    monkeypatch.setenv("RS_DEBUG_WAIT_LIMIT", "1")
    short = attend(rs, pool, q, off, ctx, n, 0.09)
    torch.cuda.synchronize()
    assert set(short[2].tolist()) <= {0, rs.RS_ST_TIMEOUT}
    for b, st in enumerate(short[2].tolist()):  # a request that reports nothing has its results
        if st == 0:
            assert torch.equal(short[0][off[b]:off[b + 1]], want[0][off[b]:off[b + 1]])
    monkeypatch.delenv("RS_DEBUG_WAIT_LIMIT")
    again = attend(rs, pool, q, off, ctx, n, 0.09)
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_calls_at_once_with_workspaces_of_their_own(rs):
    dt, D, Hkv = torch.float16, 64, 2
    lens = [5000, 700]
    pool = Pool(lens, 32, Hkv, D, 6)
    fill(rs, pool, lens, dt, 71)
    calls = []
    for i, n in enumerate((1, 4, 60, 300)):
        off, ctx = [0, n, 2 * n], [5000 - n, 700 - n]
        calls.append((rows(2 * n, 8, D, dt, 80 + i), off, ctx, n, torch.cuda.Stream()))
    alone = [attend(rs, pool, q, off, ctx, n, 0.1) for q, off, ctx, n, _ in calls]
    bufs = []
    for q, off, ctx, n, _ in calls:
        need = rs.rs_coded_attn_workspace_size(2, 2 * n, n, 8, Hkv, D)
        bufs.append((torch.empty_like(q), torch.empty(2 * n, 8, device="cuda"), i32([-1, -1]),
                     torch.empty(need, dtype=torch.uint8, device="cuda"), i32(off), pool.args(i32(ctx))))
    torch.cuda.synchronize()
    for _ in range(8):
        for (q, off, ctx, n, s), (out, lse, st, ws, offs, args) in zip(calls, bufs):
            rs.rs_coded_attn(q, 8 * D, rs.RS_F16, offs, None, 2, 2 * n, n, 8, Hkv, D, *args, 0.1, out, lse, st, ws, stream=s)
    torch.cuda.synchronize()
    for (out, lse, st, *_), want in zip(bufs, alone):
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and st.tolist() == [0, 0]


@pytest.mark.parametrize("n", [1, 2, 40])
def test_a_request_with_too_many_tokens_among_others(rs, n):
    dt, D, Hkv = torch.bfloat16, 128, 2
    ns = [n, n + 1, 0, n]
    off = [0]
    for x in ns:
        off.append(off[-1] + x)
    ctx = [200, 300, 5, 0]
    pool = Pool([c + x for c, x in zip(ctx, ns)], 16, Hkv, D, 6)
    fill(rs, pool, [c + x for c, x in zip(ctx, ns)], dt, 71)
    q = rows(off[-1], 8, D, dt, 73)
    got = attend(rs, pool, q, off, ctx, n, 0.09)
    assert got[2].tolist() == [0, rs.RS_ST_TOO_LARGE, 0, 0]
    check_attention(pool, q, off, ctx, 0.09, got, skip=[1])
    assert (got[0][off[1]:off[2]] == 0).all() and (got[1][off[1]:off[2]] == 0).all()


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_scores_of_minus_infinity_and_infinite_queries(rs, n, dt):
    """An infinite query element makes its row's scores infinite of either sign or NaN: that row is not a number, no other changes."""
    D, Hkv = 64, 2
    pool = Pool([90 + n], 16, Hkv, D, 6)
    fill(rs, pool, [90 + n], dt, 71)
    q = rows(n, 4, D, dt, 73)
    want = attend(rs, pool, q, [0, n], [90], n, 0.1)
    q[n - 1, 2, 7] = float("inf")
    got = attend(rs, pool, q, [0, n], [90], n, 0.1)
    assert got[2].tolist() == [0]
    same = torch.ones(n, 4, dtype=torch.bool, device="cuda")
    same[n - 1, 2] = False
    assert torch.equal(got[0][same], want[0][same]) and torch.equal(got[1][same], want[1][same])
    assert got[0][n - 1, 2].isnan().all() and not got[1][n - 1, 2].isfinite()


@pytest.mark.parametrize("n,most", [(1, 1), (3, 3), (40, 40)])
def test_zero_queries_and_a_scale_that_makes_one_key_all(rs, n, most):
    """Equal weights on every key; and scores so far apart that the largest takes all."""
    dt, D, Hkv = torch.bfloat16, 128, 1
    pool = Pool([500 + n], 32, Hkv, D, 6)
    fill(rs, pool, [500 + n], dt, 71, 0.0)
    q = rows(n, 2, D, dt, 73)
    got = attend(rs, pool, q * 0, [0, n], [500], most, 0.1)
    check_attention(pool, q * 0, [0, n], [500], 0.1, got)
    got = attend(rs, pool, q, [0, n], [500], most, 30.0)
    check_attention(pool, q, [0, n], [500], 30.0, got)
    at = slots(pool.table, 0, 501, 32)
    assert len(set(at.tolist())) == 501


@pytest.mark.parametrize("B,most,ctx_lo,ctx_hi,Hq,Hkv,D,tree,dt", [
    (25, 4, 0, 0, 64, 16, 128, False, torch.float16), (6, 4, 0, 0, 40, 40, 128, True, torch.bfloat16), (24, 1, 18, 150, 16, 16, 128, True, torch.bfloat16),
    (700, 1, 0, 50, 8, 4, 64, False, torch.bfloat16), (60, 8, 30, 90, 6, 6, 64, True, torch.float16), (33, 2, 0, 40, 15, 5, 128, False, torch.float16)])
def test_many_short_requests(rs, B, most, ctx_lo, ctx_hi, Hq, Hkv, D, tree, dt):
    """Segments of a few blocks, fewer and more than there are CTAs; some requests without tokens."""
    g = random.Random(B)
    ns = [g.randrange(0 if b % 7 == 3 else 1, most + 1) for b in range(B)]
    ctx = [g.randrange(ctx_lo, ctx_hi + 1) for _ in range(B)]
    off = [0]
    for x in ns:
        off.append(off[-1] + x)
    lens = [c + x for c, x in zip(ctx, ns)]
    pool = Pool(lens, 16, Hkv, D, 5)
    fill(rs, pool, lens, dt, 21)
    q = rows(off[-1] + 1, Hq, D, dt, 23)
    parents = i32([-1 if i == 0 else g.randrange(i) for x in ns for i in range(x)] + [0]) if tree else None
    got = attend(rs, pool, q, off, ctx, most, D ** -0.5, parents)
    check_attention(pool, q, off, ctx, D ** -0.5, got, parents)
    assert (got[0][-1:] == 7).all() and (got[1][-1:] == 7).all()


def seen_keys(ctx, n, parents=None):
    see = causal_mask(n, ctx)
    return see if parents is None else torch.cat([torch.ones(n, ctx, dtype=torch.bool), tree_mask(parents)], 1)


# (Hq, Hkv, D, page, ctx, ns): few rows with heads apart (caches of 100 tokens and more) and side by side (shorter ones, and many
# heads), one, two and four tiles of eight rows; and many rows, of one and two row tiles, of trees over three runs of 128 slots
@pytest.mark.parametrize("Hq,Hkv,D,page,ctx,ns,dt", [
    (1, 1, 64, 16, [12], [8], torch.float16), (4, 4, 128, 16, [12, 30], [8, 7], torch.bfloat16), (2, 2, 64, 32, [300, 0, 1000], [5, 8, 2], torch.bfloat16),
    (8, 2, 128, 64, [140, 5], [4, 3], torch.float16), (4, 2, 64, 16, [15, 47], [16, 9], torch.float16), (8, 2, 128, 16, [250, 3], [8, 8], torch.bfloat16),
    (1, 1, 128, 32, [7, 100, 2000], [32, 20, 31], torch.float16), (2, 1, 64, 16, [14], [16], torch.bfloat16),
    (4, 4, 64, 16, [60, 129], [200, 65], torch.float16), (8, 2, 128, 64, [100, 5000], [256, 33], torch.bfloat16), (2, 2, 128, 32, [64], [256], torch.float16),
    (8, 2, 64, 128, [20000], [250], torch.bfloat16), (3, 1, 64, 32, [0, 500], [256, 90], torch.bfloat16)])
@pytest.mark.parametrize("tree", [False, True])
def test_nan_in_new_tokens_reaches_the_rows_that_see_it(rs, Hq, Hkv, D, page, ctx, ns, dt, tree):
    """NaN in V of some of the new tokens and of the last cached one, in columns of their own: there the rows that see the token,
    nothing else of any row."""
    off = [0]
    for x in ns:
        off.append(off[-1] + x)
    lens = [c + x for c, x in zip(ctx, ns)]
    pool = Pool(lens, page, Hkv, D, 5)
    fill(rs, pool, lens, dt, 21)
    q = rows(off[-1], Hq, D, dt, 23)
    g = random.Random(7)
    # (node 3 begins a branch that the root's other children do not see)
    tops = [[-1 if i == 0 else 0 if i < 6 else g.randrange(i) for i in range(x)] for x in ns]
    parents = i32([p for t in tops for p in t]) if tree else None
    want = attend(rs, pool, q, off, ctx, max(ns), 0.11, parents)
    check_attention(pool, q, off, ctx, 0.11, want, parents)
    nans = torch.zeros(off[-1], Hq, D, dtype=torch.bool)
    for b, n in enumerate(ns):
        see = seen_keys(ctx[b], n, tops[b] if tree else None)
        at = slots(pool.table, b, lens[b], page)
        for node, h, col, code in ((n - 1, 0, 3, 0x7f), (n // 2, Hkv - 1, D - 1, 0xff), (min(3, n - 1), 0, D // 2 + 1, 0x7f), (n - 1, Hkv - 1, 40, 0xff)):
            pool.v.view(-1, Hkv, D)[at[ctx[b] + node], h, col] = code
            nans[off[b]:off[b + 1], h * Hq // Hkv:(h + 1) * Hq // Hkv, col] |= see[:, ctx[b] + node, None]
        if ctx[b]:  # the last cached token is for all rows
            pool.v.view(-1, Hkv, D)[at[ctx[b] - 1], 0, 20] = 0x7f
            nans[off[b]:off[b + 1], :Hq // Hkv, 20] = True
    got = attend(rs, pool, q, off, ctx, max(ns), 0.11, parents)
    nans = nans.cuda()
    assert got[2].tolist() == [0] * len(ns) and torch.equal(got[1], want[1])
    assert torch.equal(got[0].isnan(), nans), (got[0].isnan() != nans).nonzero()[:5]
    assert torch.equal(got[0][~nans], want[0][~nans])
    # NaN in K: whole rows
    fill(rs, pool, lens, dt, 21)
    whole = torch.zeros(off[-1], Hq, dtype=torch.bool)
    for b, n in enumerate(ns):
        at = slots(pool.table, b, lens[b], page)
        for node in (n - 1, min(3, n - 1)):
            pool.k.view(-1, Hkv, D)[at[ctx[b] + node], Hkv - 1, 9] = 0x7f
            whole[off[b]:off[b + 1], (Hkv - 1) * Hq // Hkv:] |= seen_keys(ctx[b], n, tops[b] if tree else None)[:, ctx[b] + node, None]
    got = attend(rs, pool, q, off, ctx, max(ns), 0.11, parents)
    whole = whole.cuda()
    assert got[2].tolist() == [0] * len(ns) and torch.equal(got[1].isnan(), whole) and got[0][whole].isnan().all()
    assert torch.equal(got[0][~whole], want[0][~whole]) and torch.equal(got[1][~whole], want[1][~whole])


@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lo,hi", [(-117, -105), (113, 120)])
def test_the_smallest_and_largest_values(rs, n, D, lo, hi):
    dt, Hkv = torch.bfloat16, 2
    pool = Pool([400], 32, Hkv, D, 9)
    fill(rs, pool, [400], dt, 41, 0.0)
    g = torch.Generator().manual_seed(1)
    pool.ve = torch.randint(lo, hi + 1, pool.ve.shape, generator=g).to(torch.int8).cuda()
    pool.v &= 0xbf  # (codes of 2^8 at exponent 120 are above bf16)
    q = rows(n, 2 * Hkv, D, dt, 43) * 3
    got = attend(rs, pool, q, [0, n], [400 - n], n, 0.125)
    check_attention(pool, q, [0, n], [400 - n], 0.125, got)


@pytest.mark.parametrize("n", [1, 8, 40])
def test_the_smallest_values_behind_larger_ones(rs, n):
    """Keys of weight 1 and values near 2^-105, 128 slots on some of weight 2^18.75 and values near 2^-117, others of no weight: the first
    bound the products, the second the weights, and the quotient of the two bounds is below fp32's normal numbers."""
    dt, D, page, N = torch.bfloat16, 64, 16, 400
    pool = Pool([N], page, 1, D, 9)
    fill(rs, pool, [N], dt, 41, 0.0)
    at = slots(pool.table, 0, N, page)
    k, ve = pool.k.view(-1, 1, D), pool.ve.view(-1)
    k[at] = 0
    k[at[16:], 0, 0] = 0xe0  # -32
    k[at[128:160], 0, 0] = 0x55  # 13
    pool.ke.zero_()
    ve[:] = -117
    ve[at[0] // 16] = -105
    q = torch.zeros(n, 2, D, dtype=dt, device="cuda")
    q[..., 0] = 1.0
    got = attend(rs, pool, q, [0, n], [N - n], n, 1.0)
    check_attention(pool, q, [0, n], [N - n], 1.0, got)
    assert (got[0] != 0).float().mean() > 0.9


@pytest.mark.parametrize("n", [1, 8, 40])
def test_a_score_below_all_numbers_beside_zeros(rs, n):
    """q.k of -2^240 at one key of a block and 0 at the others, whose factors are above fp32's largest number: equal weights on these."""
    dt, D, page, N = torch.bfloat16, 64, 16, 200
    pool = Pool([N], page, 1, D, 9)
    v = rows(N, 1, D, dt, 42)
    k = torch.zeros_like(v)
    k[5, 0, 7] = -2.0 ** 120
    assert append(rs, pool, k, v, [0, N], [0]) == [0]
    q = torch.zeros(n, 2, D, dtype=dt, device="cuda")
    q[..., 7] = 2.0 ** 120
    out, lse, st = attend(rs, pool, q, [0, n], [N - n], n, 0.125)
    assert st.tolist() == [0]
    at = slots(pool.table, 0, N, page)
    val = cr.values(pool.v, pool.ve).view(-1, D).cuda()[at]
    for i in range(n):
        on = torch.arange(N - n + i + 1) != 5
        mean = val[:N - n + i + 1][on].mean(0)
        tol = (2.0 ** -9 + 2.0 ** -10) * (mean.abs() + val.abs().mean(0) * 1.1)  # out's rounding, P's
        assert ((out[i].double() - mean).abs() <= tol).all()
        assert (lse[i] - math.log(N - n + i)).abs().max() <= 2.0 ** -18


@pytest.mark.parametrize("n", [1, 300])
def test_a_wait_that_has_run_out_is_in_the_status(rs, n, monkeypatch):
    """With a limit of one cycle some wait does run out (of single tokens most calls have one, of chunks every request), and says so;
    a request that says nothing has all of its results."""
    dt, D, Hkv, B = torch.bfloat16, 128, 8, 8
    lens = [20000 + n] * B
    pool = Pool(lens, 64, Hkv, D, 6)
    fill(rs, pool, lens, dt, 71)
    ctx, off = [20000] * B, [i * n for i in range(B + 1)]
    q = rows(B * n, 32, D, dt, 73)
    want = attend(rs, pool, q, off, ctx, n, 0.09)
    assert want[2].tolist() == [0] * B
    monkeypatch.setenv("RS_DEBUG_WAIT_LIMIT", "1")
    told = 0
    for _ in range(20):
        out, lse, status = attend(rs, pool, q, off, ctx, n, 0.09)
        status = status.tolist()
        assert set(status) <= {0, rs.RS_ST_TIMEOUT}
        told += sum(s != 0 for s in status)
        for b, s in enumerate(status):
            a = slice(off[b], off[b + 1])
            assert s or (torch.equal(out[a], want[0][a]) and torch.equal(lse[a], want[1][a]))
        if told:
            break
    assert told
    monkeypatch.delenv("RS_DEBUG_WAIT_LIMIT")
    again = attend(rs, pool, q, off, ctx, n, 0.09)
    assert all(torch.equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("n", [1, 8, 40])
def test_rejected_ranges_leave_all_rows_but_the_others(rs, n):
    dt, D, Hkv = torch.bfloat16, 64, 2
    lens = [100] * 4
    pool = Pool(lens, 16, Hkv, D, 6)
    fill(rs, pool, lens, dt, 71)
    ctx, q = [100 - n] * 4, rows(4 * n, 4, D, dt, 73)
    for off, bad in (([0, n, 4 * n + 1, 4 * n + 1, 4 * n + 1], [1, 2, 3]), ([n, 2 * n, n, 2 * n, 3 * n], [1, 2]), ([-1, n, 2 * n, 2 * n, 3 * n], [0])):
        got = attend(rs, pool, q, off, ctx, n, 0.125)
        assert [s == rs.RS_ST_BAD_OFFSET for s in got[2].tolist()] == [b in bad for b in range(4)]
        check_attention(pool, q, off, ctx, 0.125, got, skip=bad)
        mine = torch.zeros(4 * n, dtype=torch.bool, device="cuda")
        for b in set(range(4)) - set(bad):
            mine[off[b]:off[b + 1]] = True
        assert (got[0][~mine] == 7).all() and (got[1][~mine] == 7).all() and not mine.all()
