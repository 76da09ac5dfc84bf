"""What the prompt and paged-cache calls do with bad device data, odd values, other streams, graphs and limits."""
import os

import pytest
import torch

from paged_ref import attention, causal_mask, check, slots, weights as ref_weights
from paper_2511_01282_gb300 import respec as rs
from test_gpu_evict import evict, weigh
from test_gpu_prompt_paged import DT, _i32, _normal, _off, _pool, _scratch, append, run_paged, run_prompt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _qkv(T, Hq, Hkv, D, dt=torch.bfloat16, seed=0):
    return _normal(seed, T, Hq, D, dtype=dt), _normal(seed + 1, T, Hkv, D, dtype=dt), _normal(seed + 2, T, Hkv, D, dtype=dt)


def _same(q, k, v, out, lse, a, e, scale):
    o, z, o_tol, z_tol = attention(q[a:e], k[a:e], v[a:e], causal_mask(e - a, 0), scale)
    check(out[a:e], o, o_tol, "out")
    check(lse[a:e], z, z_tol, "lse")


@pytest.mark.parametrize("off,bad", [
    ([0, 50, 30, 100], [1, 2]),    # ends before it starts; starts before an earlier one
    ([0, 50, 500, 100], [1, 2]),   # ends outside; starts outside
    ([-5, 50, 60, 100], [0]),
    ([0, 100, 0, 100], [1, 2]),
])
def test_prompt_bad_offsets(off, bad):
    q, k, v = _qkv(100, 8, 2, 64)
    out, lse, status = run_prompt(q, k, v, off, rs.RS_BF16, 0.125)
    assert [b for b in range(3) if status[b]] == bad and all(int(status[b]) == rs.RS_ST_BAD_OFFSET for b in bad)
    good = [b for b in range(3) if b not in bad]
    for b in good:
        _same(q, k, v, out, lse, off[b], off[b + 1], 0.125)
    rows = torch.zeros(100, dtype=torch.bool)
    for b in good:
        rows[off[b]:off[b + 1]] = True
    rest = out[~rows.cuda()].float()
    assert bool(((rest == 0) | (rest == 7)).all())  # emptied, or nobody's


def _cache(n, ctx, page, Hkv=2, D=64, dt=torch.bfloat16):
    pages, most, table, kp, vp = _pool(n, ctx, page, Hkv, D, dt, 3)
    kp, vp = _normal(7, *kp.shape, dtype=dt), _normal(8, *vp.shape, dtype=dt)
    return pages, most, table, kp, vp


def test_paged_bad_requests():
    n, ctx, page, Hq, Hkv, D = [3, 3, 3, 3, 3], [100, 100, 100, 100, 100], 16, 4, 2, 64
    pages, most, table, kp, vp = _cache(n, ctx, page)
    off = _off(n)
    q = _normal(1, off[-1], Hq, D, dtype=torch.bfloat16)
    table[1, 2] = pages          # outside the pool
    table[2, 5] = -1
    bad_ctx = [100, 100, 100, most * page - 2, -1]  # more slots than pages; negative
    k0 = kp.clone()
    out, lse, status = run_paged(q, rs.RS_BF16, off, None, kp, vp, page, table, bad_ctx, 0.125)
    want = [0, rs.RS_ST_BAD_PAGE, rs.RS_ST_BAD_PAGE, rs.RS_ST_BAD_OFFSET, rs.RS_ST_BAD_OFFSET]
    assert status.tolist() == want
    assert bool((out[3:] == 0).all()) and bool((lse[3:] == 0).all())
    at = slots(table, 0, 103, page)
    o, z, o_tol, z_tol = attention(q[:3], kp.view(-1, Hkv, D)[at], vp.view(-1, Hkv, D)[at], causal_mask(3, 100), 0.125)
    check(out[:3], o, o_tol, "out")
    # append: nothing outside the good pages is written
    nk = torch.full((15, Hkv, D), 5.0, dtype=torch.bfloat16, device="cuda")
    table[1, 6] = 1 << 29        # the page of the new tokens
    st = append(nk, nk, None, off, kp, vp, page, table, bad_ctx)
    assert st.tolist() == [0, rs.RS_ST_BAD_PAGE, 0, rs.RS_ST_BAD_OFFSET, rs.RS_ST_BAD_OFFSET]
    written = (kp.view(-1, Hkv, D) != k0.view(-1, Hkv, D)).any(-1).any(-1)
    good = torch.cat([slots(table, b, 103, page)[100:] for b in (0, 2)])
    assert set(torch.nonzero(written).flatten().tolist()) == set(good.tolist())
    # weights: the same for every key in a good page
    w = torch.zeros(Hkv, pages * page, device="cuda")
    st = weigh(q, rs.RS_BF16, torch.ones(15, Hq, device="cuda"), off, kp, page, table, bad_ctx, 0.125, w)
    assert st.tolist() == want
    assert bool((w[:, slots(table, 0, 103, page)] > 0).all())
    # eviction: a request with a bad page, or too long, is left alone
    pos = torch.zeros(Hkv, pages * page, dtype=torch.int32, device="cuda")
    k1, w1 = kp.clone(), w.clone()
    new, st = evict(kp, vp, page, table, [103, 103, 103, most * page + 1, -4], [200] * 5, 50, 0, w, pos)
    assert st == want and new == [50, 103, 103, most * page + 1, -4]
    keep = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    keep[slots(table, 0, 103, page)[:50]] = False
    assert torch.equal(kp.view(-1, Hkv, D)[keep], k1.view(-1, Hkv, D)[keep]) and torch.equal(w[:, keep], w1[:, keep])


def test_append_rejects_offsets_that_decrease():
    n, ctx, page = [4, 4], [0, 0], 8
    pages, most, table, kp, vp = _cache(n, ctx, page)
    k0 = kp.clone()
    nk = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    for off in ([0, 6, 4], [-1, 4, 8], [0, 4, 9]):
        st = append(nk, nk, None, off, kp, vp, page, table, ctx)
        assert st.tolist() == [rs.RS_ST_BAD_OFFSET] * 2 and torch.equal(kp, k0)


def test_bad_trees():
    n, ctx, page, Hq, Hkv, D = [5, 5, 300, 5], [20, 20, 20, 0], 16, 4, 2, 64
    pages, most, table, kp, vp = _cache(n, ctx, page)
    off = _off(n)
    q = _normal(1, off[-1], Hq, D, dtype=torch.bfloat16)
    par = [-1, 0, 1, 3, 0] + [0, 0, 0, 0, 0] + [-1] + [0] * 299 + [-1, 0, 1, 2, 3]
    out, lse, status = run_paged(q, rs.RS_BF16, off, _i32(par), kp, vp, page, table, ctx, 0.125)
    assert status.tolist() == [rs.RS_ST_BAD_TREE, rs.RS_ST_BAD_TREE, rs.RS_ST_TOO_LARGE, 0]
    assert bool((out[:310] == 0).all()) and bool((lse[:310] == 0).all())
    a, at = 310, slots(table, 3, 5, page)
    o, z, o_tol, z_tol = attention(q[a:], kp.view(-1, Hkv, D)[at], vp.view(-1, Hkv, D)[at], causal_mask(5, 0), 0.125)
    check(out[a:], o, o_tol, "a chain is causal")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_large_and_odd_values(D, t):
    """Scores of hundreds, rows that only see -inf, infinities and NaN that reach their own sequence only."""
    dt, code = DT[t]
    n = [300, 200, 150, 130]
    off = _off(n)
    q, k, v = _qkv(off[-1], 4, 2, D, dt)
    q[:300] *= 20.0                       # scores to several hundred: the maximum moves all the time
    k[100] *= 30.0
    q[300:500], k[300:500] = 60.0, -60.0  # every score far below zero, all equal
    k[500:650] = float("-inf")            # 3 is the sequence whose scores are all -inf or NaN
    q[500:650] = q[500:650].abs() + 0.1
    v[650 + 64] = float("nan")            # 4: NaN at one key, from its tile on
    out, lse, status = run_prompt(q, k, v, off, code, D ** -0.5)
    assert status.tolist() == [0] * 4
    for a, e in ((0, 300), (300, 500)):
        _same(q, k, v, out, lse, a, e, D ** -0.5)
    assert bool((out[500:650] == 0).all()) and bool(torch.isneginf(lse[500:650]).all())
    assert bool(out[650 + 64:].isnan().all()) and bool(torch.isfinite(lse[650:]).all())


def test_scores_of_one_sequence_do_not_reach_another():
    """Every other sequence is NaN throughout; pages behind the last token too."""
    n = [70, 65, 3, 128, 40]
    off = _off(n)
    q, k, v = _qkv(off[-1], 6, 2, 128, torch.float16)
    for b in (1, 3):
        for x in (q, k, v):
            x[off[b]:off[b + 1]] = float("nan")
    out, lse, status = run_prompt(q, k, v, off, rs.RS_F16, 0.09)
    for b in (0, 2, 4):
        _same(q, k, v, out, lse, off[b], off[b + 1], 0.09)
    for b in (1, 3):
        assert bool(out[off[b]:off[b + 1]].isnan().all())


def test_a_steep_climb_of_the_maximum():
    """Keys in ascending order of their scores, by a little and by a lot: O is rescaled at every tile, in both halves."""
    D, T = 128, 1500
    for step in (0.02, 0.4, 3.0):
        q = torch.full((T, 2, D), 1.0, dtype=torch.bfloat16, device="cuda")
        k = torch.zeros(T, 2, D, dtype=torch.bfloat16, device="cuda")
        k[:, :, 0] = (torch.arange(T, device="cuda") * step)[:, None]
        v = _normal(3, T, 2, D, dtype=torch.bfloat16)
        out, lse, _ = run_prompt(q, k, v, [0, T], rs.RS_BF16, 1.0)
        _same(q, k, v, out, lse, 0, T, 1.0)


def test_graph_replay_with_new_data():
    n, ctx, page, Hq, Hkv, D = [1, 4, 70], [40, 300, 10], 16, 8, 2, 128
    dt, code = DT["bf16"]
    pages, most, table, kp, vp = _cache(n, ctx, page, Hkv, D)
    off = _off(n)
    T, B, S = off[-1], 3, pages * page
    q, k, v = _qkv(T, Hq, Hkv, D)
    out, lse = torch.zeros(T, Hq, D, dtype=dt, device="cuda"), torch.zeros(T, Hq, device="cuda")
    p_out, p_lse = torch.zeros_like(out), torch.zeros_like(lse)
    status, new = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    w, pos = torch.zeros(Hkv, S, device="cuda"), torch.zeros(Hkv, S, dtype=torch.int32, device="cuda")
    need = max(rs.rs_prompt_attn_workspace_size(B, T, Hq, Hkv, D), rs.rs_paged_attn_workspace_size(B, T, Hq, Hkv, D),
               rs.rs_paged_weights_workspace_size(B, T, Hq, Hkv, D), rs.rs_paged_evict_workspace_size(B, Hkv, 32))
    ws = _scratch(need)
    o_dev, c_dev, l_dev = _i32(off), _i32(ctx), _i32([a + c for a, c in zip(n, ctx)])

    def step():
        rs.rs_prompt_attn(q, Hq * D, k, Hkv * D, v, Hkv * D, code, o_dev, B, T, Hq, Hkv, D, 0.09, p_out, p_lse, status, ws)
        rs.rs_paged_append(k, Hkv * D, v, Hkv * D, None, o_dev, B, T, Hkv, D, kp, vp, pages, page, table, most, c_dev, w, pos, status)
        rs.rs_paged_attn(q, Hq * D, code, o_dev, None, B, T, Hq, Hkv, D, kp, vp, pages, page, table, most, c_dev, 0.09, out, lse, status, ws)
        rs.rs_paged_weights(q, Hq * D, code, lse, o_dev, B, T, Hq, Hkv, D, kp, pages, page, table, most, c_dev, 0.09, w, status, ws)
        rs.rs_paged_evict(kp, vp, Hkv, D, pages, page, table, most, l_dev, l_dev, B, 32, 4, w, pos, new, status, ws)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    results = []
    for seed in (5, 6):  # the second replay on other data, and once eagerly on the same
        fresh = _qkv(T, Hq, Hkv, D, seed=seed) + (_normal(90 + seed, *kp.shape, dtype=dt), _normal(91 + seed, *vp.shape, dtype=dt))
        got = []
        for run in (g.replay, step):
            for x, y in zip((q, k, v, kp, vp), fresh):
                x.copy_(y)
            w.zero_()
            pos.zero_()
            run()
            torch.cuda.synchronize()
            got.append([x.clone() for x in (p_out, p_lse, out, lse, w, pos, kp, vp, new)])
        for x, y in zip(*got):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        results.append(got[0])
    assert not torch.equal(results[0][2], results[1][2])


def test_another_stream_and_two_calls_at_once():
    """Two streams with a workspace each, at the same time, give what each gives alone."""
    q, k, v = _qkv(900, 8, 2, 128)
    alone = [run_prompt(q[a:], k[a:], v[a:], [0, 900 - a], rs.RS_BF16, 0.09) for a in (0, 300)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = []
    for a in (0, 300):
        T = 900 - a
        bufs.append((torch.zeros(T, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 8, device="cuda"),
                     torch.zeros(1, dtype=torch.int32, device="cuda"), _scratch(rs.rs_prompt_attn_workspace_size(1, T, 8, 2, 128)),
                     _i32([0, T])))
    torch.cuda.synchronize()
    for _ in range(5):
        for a, st, (out, lse, status, ws, off) in zip((0, 300), streams, bufs):
            rs.rs_prompt_attn(q[a:], 1024, k[a:], 256, v[a:], 256, rs.RS_BF16, off, 1, 900 - a, 8, 2, 128, 0.09, out, lse, status, ws,
                              stream=st)
    torch.cuda.synchronize()
    for (out, lse, status, *_), want in zip(bufs, alone):
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and status.tolist() == [0]


def test_waits_that_run_out_report_it(monkeypatch):
    """A limit of one cycle: the pipelines give up, say so, and the next call works.  (A try to pass a barrier itself waits for
    some microseconds, so the calls have to be long enough for one to fail.)"""
    T = 5000
    q, k, v = _qkv(T, 32, 8, 128)
    monkeypatch.setenv("RS_DEBUG_WAIT_LIMIT", "1")
    _, _, status = run_prompt(q, k, v, [0, T], rs.RS_BF16, 0.09)
    torch.cuda.synchronize()
    assert status.tolist() == [rs.RS_ST_TIMEOUT]
    pages, most, table, kp, vp = _cache([T], [20], 16, 8, 128)
    w = torch.zeros(8, pages * 16, device="cuda")
    lse = torch.full((T, 32), 5.0, device="cuda")
    st = weigh(q, rs.RS_BF16, lse, [0, T], kp, 16, table, [20], 0.09, w)
    torch.cuda.synchronize()
    assert st.tolist() == [rs.RS_ST_TIMEOUT]
    monkeypatch.delenv("RS_DEBUG_WAIT_LIMIT")
    out, lse, status = run_prompt(q, k, v, [0, T], rs.RS_BF16, 0.09)
    assert status.tolist() == [0]
    _same(q, k, v, out, lse, 0, T, 0.09)


def test_many_requests():
    """As many as a call takes, most of them empty or of one token."""
    B = 4096
    n = [(i * 7) % 3 if i % 100 else 150 for i in range(B)]
    off = _off(n)
    q, k, v = _qkv(off[-1], 2, 1, 64)
    out, lse, status = run_prompt(q, k, v, off, rs.RS_BF16, 0.125)
    assert not bool(status.any())
    for b in (0, 1, 2, 100, 101, 2047, 4000, 4094, 4095):
        if n[b]:
            _same(q, k, v, out, lse, off[b], off[b + 1], 0.125)
    one = [1] * B
    ctx = [(i * 13) % 50 for i in range(B)]
    pages, most, table, kp, vp = _cache(one, ctx, 8, 1, 64)
    q = _normal(1, B, 2, 64, dtype=torch.bfloat16)
    out, lse, status = run_paged(q, rs.RS_BF16, _off(one), None, kp, vp, 8, table, ctx, 0.125)
    assert not bool(status.any())
    for b in (0, 1, 49, 50, 3000, 4095):
        at = slots(table, b, ctx[b] + 1, 8)
        o, z, o_tol, z_tol = attention(q[b:b + 1], kp.view(-1, 1, 64)[at], vp.view(-1, 1, 64)[at], causal_mask(1, ctx[b]), 0.125)
        check(out[b:b + 1], o, o_tol, "request %d" % b)
    w = torch.zeros(1, pages * 8, device="cuda")
    st = weigh(q, rs.RS_BF16, lse, _off(one), kp, 8, table, ctx, 0.125, w)
    assert not bool(st.any())
    for b in (0, 1, 49, 50, 3000, 4095):
        at = slots(table, b, ctx[b] + 1, 8)
        want, tol = ref_weights(q[b:b + 1], kp.view(-1, 1, 64)[at], lse[b:b + 1], causal_mask(1, ctx[b]), 0.125)
        check(w[:, at], want, tol + 1e-30, "weights of request %d" % b)


def test_a_long_cache():
    """One request of 300000 tokens: weights and eviction past what shared memory holds, slots far behind."""
    n, ctx, page, Hkv, D = [2], [300000], 256, 1, 64
    pages, most, table, kp, vp = _cache(n, ctx, page, Hkv, D)
    q = _normal(1, 2, 4, D, dtype=torch.bfloat16) * 2.0
    out, lse, status = run_paged(q, rs.RS_BF16, [0, 2], None, kp, vp, page, table, ctx, 0.125)
    at = slots(table, 0, ctx[0] + 2, page)
    K, V = kp.view(-1, Hkv, D)[at], vp.view(-1, Hkv, D)[at]
    o, z, o_tol, z_tol = attention(q, K, V, causal_mask(2, ctx[0]), 0.125)
    check(out, o, o_tol, "out")
    check(lse, z, z_tol, "lse")
    w = torch.zeros(Hkv, pages * page, device="cuda")
    assert weigh(q, rs.RS_BF16, lse, [0, 2], kp, page, table, ctx, 0.125, w).tolist() == [0]
    want, tol = ref_weights(q, K, lse, causal_mask(2, ctx[0]), 0.125)
    check(w[:, at], want, tol, "weights")
    pos = torch.zeros(Hkv, pages * page, dtype=torch.int32, device="cuda")
    pos[0, at] = torch.arange(len(at), dtype=torch.int32, device="cuda")
    w0 = w[0, at].clone()
    new, st = evict(kp, vp, page, table, [300002], [300002], 1000, 100, w, pos)
    assert new == [1000] and st == [0]
    key = w0.clone()
    key[-100:] = float("inf")
    kept = set(torch.sort(key, descending=True, stable=True).indices[:1000].tolist())
    assert set(pos[0, at[:1000]].tolist()) == kept
    assert torch.equal(kp.view(-1, Hkv, D)[at[:1000], 0], K[pos[0, at[:1000]].long(), 0])


FIRST = """
import sys, torch
sys.path[:0] = [%r, %r]
from paper_2511_01282_gb300 import respec as rs
dev, bf = "cuda", torch.bfloat16
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
q, k, v = (torch.randn(40, h, 128, device=dev).to(bf) for h in (4, 2, 2))
kp, vp = torch.zeros(8, 16, 2, 128, dtype=bf, device=dev), torch.zeros(8, 16, 2, 128, dtype=bf, device=dev)
table, off, ctx, length = i32([[3, 1, 7, 5]]), i32([0, 40]), i32([0]), i32([40])
out, lse, st = torch.zeros(40, 4, 128, dtype=bf, device=dev), torch.zeros(40, 4, device=dev), i32([-1])
out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
w, pos, new = torch.zeros(2, 128, device=dev), torch.zeros(2, 128, dtype=torch.int32, device=dev), i32([0])
ws = torch.empty(1 << 28, dtype=torch.uint8, device=dev)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    rs.rs_prompt_attn(q, 512, k, 256, v, 256, 0, off, 1, 40, 4, 2, 128, 0.09, out, lse, st, ws)
    rs.rs_paged_append(k, 256, v, 256, None, off, 1, 40, 2, 128, kp, vp, 8, 16, table, 4, ctx, w, pos, st)
    rs.rs_paged_attn(q, 512, 0, off, None, 1, 40, 4, 2, 128, kp, vp, 8, 16, table, 4, ctx, 0.09, out2, lse2, st, ws)
    rs.rs_paged_weights(q, 512, 0, lse, off, 1, 40, 4, 2, 128, kp, 8, 16, table, 4, ctx, 0.09, w, st, ws)
    rs.rs_paged_evict(kp, vp, 2, 128, 8, 16, table, 4, length, length, 1, 20, 3, w, pos, new, st, ws)
g.replay()
torch.cuda.synchronize()
assert st.item() == 0 and new.item() == 20 and torch.equal(out, out2) and torch.equal(lse, lse2)
assert abs(float(w[:, 48:64].sum()) + float(w[:, 16:20].sum())) > 0
print("captured")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST % (root, os.path.join(root, "tests"))], capture_output=True, text=True)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_no_rows():
    q, k, v = _qkv(0, 4, 2, 64)
    out, lse, status = run_prompt(q, k, v, [0, 0, 0], rs.RS_BF16, 0.1)
    assert status.tolist() == [0, 0]
    pages, most, table, kp, vp = _cache([1, 1], [20, 30], 16)
    w = torch.ones(2, pages * 16, device="cuda")
    out, lse, status = run_paged(q, rs.RS_BF16, [0, 0, 0], None, kp, vp, 16, table, [20, 30], 0.1)
    assert status.tolist() == [0, 0]
    assert append(k, v, None, [0, 0, 0], kp, vp, 16, table, [20, 30]).tolist() == [0, 0]
    assert weigh(q, rs.RS_BF16, lse, [0, 0, 0], kp, 16, table, [20, 30], 0.1, w).tolist() == [0, 0] and bool((w == 1).all())


@pytest.mark.parametrize("Hq,Hkv", [(5, 1), (48, 4), (33, 11), (96, 2), (64, 64)])
def test_head_layouts(Hq, Hkv):
    D, n, ctx, page = 64, [37, 150], [260, 5], 32
    pages, most, table, kp, vp = _cache(n, ctx, page, Hkv, D)
    off = _off(n)
    q = _normal(1, off[-1], Hq, D, dtype=torch.bfloat16)
    out, lse, status = run_paged(q, rs.RS_BF16, off, None, kp, vp, page, table, ctx, 0.125)
    assert status.tolist() == [0, 0]
    w = torch.zeros(Hkv, pages * page, device="cuda")
    assert weigh(q, rs.RS_BF16, lse, off, kp, page, table, ctx, 0.125, w).tolist() == [0, 0]
    for b in range(2):
        a, e = off[b], off[b + 1]
        at = slots(table, b, ctx[b] + n[b], page)
        K, V, see = kp.view(-1, Hkv, D)[at], vp.view(-1, Hkv, D)[at], causal_mask(n[b], ctx[b])
        o, z, o_tol, z_tol = attention(q[a:e], K, V, see, 0.125)
        check(out[a:e], o, o_tol, "out")
        check(lse[a:e], z, z_tol, "lse")
        want, tol = ref_weights(q[a:e], K, lse[a:e], see, 0.125)
        check(w[:, at], want, tol, "weights")


def test_groups_of_heads_in_phases():
    """More keys than L2 holds, read by several pairs of row tiles each: the KV heads are worked off in groups.  Some rows of
    every head against the formula; the whole against a smaller call's bits."""
    T, Hq, Hkv, D = 72000, 8, 8, 128
    dt = torch.float16
    q, k, v = _qkv(T, Hq, Hkv, D, dt)
    out, lse, status = run_prompt(q, k, v, [0, T], rs.RS_F16, 0.09)
    assert status.tolist() == [0]
    for i in (0, 255, 256, 30000, 71999):
        o, z, o_tol, z_tol = attention(q[i:i + 1], k[:i + 1], v[:i + 1], torch.ones(1, i + 1, dtype=torch.bool), 0.09)
        check(out[i:i + 1], o, o_tol, "out of row %d" % i)
        check(lse[i:i + 1], z, z_tol, "lse of row %d" % i)
    rows = torch.arange(0, T, 977, device="cuda")
    for h in (0, 3, 7):  # one head alone: another split, the same values within both roundings
        o1, l1, _ = run_prompt(q[:, h:h + 1], k[:, h:h + 1], v[:, h:h + 1], [0, T], rs.RS_F16, 0.09)
        assert float((lse[rows, h] - l1[rows, 0]).abs().max()) < 1e-4
        assert float((out[rows, h].float() - o1[rows, 0].float()).abs().max()) < 2e-3
