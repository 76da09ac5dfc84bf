"""rs_paged_weights and rs_paged_evict against the formulas, and all five calls one after the other."""
import pytest
import torch

from paged_ref import attention, causal_mask, check, evict_order, slots, weights as ref_weights
from paper_2511_01282_gb300 import respec as rs
from test_gpu_prompt_paged import DT, _i32, _normal, _off, _pool, _scratch, append, run_paged, run_prompt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def weigh(q, code, lse, off, kp, page, table, ctx, scale, w):
    T, Hq, D = q.shape
    B, Hkv = len(off) - 1, kp.shape[2]
    status = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ws = _scratch(rs.rs_paged_weights_workspace_size(B, T, Hq, Hkv, D))
    rs.rs_paged_weights(q, q.stride(0), code, lse, _i32(off), B, T, Hq, Hkv, D, kp, kp.shape[0], page, table, table.shape[1],
                        _i32(ctx), scale, w, status, ws)
    return status


def evict(kp, vp, page, table, length, nxt, budget, recent, w, pos):
    B, Hkv, D = table.shape[0], kp.shape[2], kp.shape[3]
    status = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    new = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ws = _scratch(rs.rs_paged_evict_workspace_size(B, Hkv, budget))
    rs.rs_paged_evict(kp, vp, Hkv, D, kp.shape[0], page, table, table.shape[1], _i32(length), _i32(nxt), B, budget, recent, w, pos,
                      new, status, ws)
    return new.tolist(), status.tolist()


WEIGH = [
    # new, cached, Hq, Hkv, D, type, page
    ([1], [0], 1, 1, 64, "bf16", 8),
    ([1, 1, 1], [0, 127, 128], 8, 2, 128, "f16", 16),
    ([1, 0, 1], [5000, 300, 77], 32, 8, 128, "bf16", 64),
    ([130, 3], [200, 0], 4, 4, 128, "bf16", 128),
    ([300, 1, 64], [1000, 2500, 130], 8, 2, 64, "bf16", 8),
    ([129, 700], [300, 0], 6, 2, 128, "f16", 256),
    ([90], [33], 7, 1, 64, "f16", 32),
    ([1500], [0], 3, 1, 128, "bf16", 16),
    ([40], [300], 128, 1, 64, "bf16", 64),
]


@pytest.mark.parametrize("n,ctx,Hq,Hkv,D,t,page", WEIGH)
def test_weights(n, ctx, Hq, Hkv, D, t, page):
    dt, code = DT[t]
    scale = D ** -0.5
    pages, most, table, kp, vp = _pool(n, ctx, page, Hkv, D, dt, 3)
    S = pages * page
    off = _off(n)
    w0 = torch.rand(Hkv, S, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    w, want, tol = w0.clone(), w0.double(), torch.zeros(Hkv, S, dtype=torch.float64, device="cuda")
    q = _normal(1, off[-1] + 2, Hq, D, dtype=dt)
    q[off[-1]:] = float("nan")  # rows behind the last request
    lse = torch.full((off[-1] + 2, Hq), float("nan"), device="cuda")
    for b in range(len(n)):
        at = slots(table, b, ctx[b] + n[b], page)
        K = _normal(20 + b, len(at), Hkv, D, dtype=dt)
        kp.view(S, Hkv, D)[at] = K
        see = causal_mask(n[b], ctx[b])
        a, e = off[b], off[b + 1]
        if a == e:
            continue
        lse[a:e] = attention(q[a:e], K, K, see, scale)[1].float()
        if n[b] > 60:  # rows that count for nothing, one of them with NaN for a query
            lse[a + 3, 0], lse[a + 4, Hq - 1], lse[a + 5, 0] = float("-inf"), float("inf"), float("nan")
            q[a + 5, 0] = float("nan")
        qq = torch.where(q[a:e].isnan(), torch.zeros((), dtype=dt, device="cuda"), q[a:e])
        got, t_b = ref_weights(qq, K, lse[a:e], see, scale)
        want[:, at] += got
        tol[:, at] += t_b + 2.0 ** -23 * (want[:, at])
    assert weigh(q, code, lse, off, kp, page, table, ctx, scale, w).tolist() == [0] * len(n)
    check(w, want, tol, "weights")
    again = w0.clone()
    weigh(q, code, lse, off, kp, page, table, ctx, scale, again)
    assert torch.equal(again, w)


EVICT = [
    # lengths, budget, recent, Hkv, D, page
    ([5, 1, 0], 1, 0, 1, 64, 8),
    ([300, 299, 301], 300, 20, 2, 128, 16),
    ([2500, 100, 1025], 700, 700, 3, 64, 32),
    ([4000], 64, 10, 8, 128, 64),
    ([1024, 2048, 2049], 1024, 1, 1, 128, 256),
    ([9000, 40], 2500, 0, 2, 64, 8),
]


@pytest.mark.parametrize("length,budget,recent,Hkv,D,page", EVICT)
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(length, budget, recent, Hkv, D, page, kind):
    B = len(length)
    pages, most, table, kp, vp = _pool(length, [0] * B, page, Hkv, D, torch.bfloat16, 8)
    S = pages * page
    g = torch.Generator(device="cuda").manual_seed(budget)
    bits = lambda: torch.randint(-32768, 32767, kp.shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)  # noqa: E731
    kp, vp = bits(), bits()
    w = torch.randn(Hkv, S, generator=g, device="cuda")
    if kind == "ties":
        w = (w * 1.5).round()
    if kind == "odd":
        for i, x in enumerate((float("inf"), float("-inf"), float("nan"), 0.0, -0.0, 1e-45, 3.4e38)):
            w[:, i::11] = x
    pos = torch.stack([torch.randperm(S, generator=g, device="cuda") for _ in range(Hkv)]).int()
    nxt = [S - S // 3 + b for b in range(B)]  # positions at or behind next_pos - recent are recent, however many
    k0, v0, w0, pos0 = (x.clone() for x in (kp, vp, w, pos))
    new, status = evict(kp, vp, page, table, length, nxt, budget, recent, w, pos)
    assert new == [min(x, budget) for x in length] and status == [0] * B
    for b in range(B):
        at = slots(table, b, length[b], page)
        if length[b] <= budget:
            continue
        for h in range(Hkv):
            for src, dst in evict_order(w0[h, at].tolist(), pos0[h, at].tolist(), nxt[b], recent, budget):
                a, d = int(at[src]), int(at[dst])
                k0.view(S, Hkv, D)[d, h] = k0.view(S, Hkv, D)[a, h]
                v0.view(S, Hkv, D)[d, h] = v0.view(S, Hkv, D)[a, h]
                w0[h, d], pos0[h, d] = w0[h, a], pos0[h, a]
    same = lambda x, y: torch.equal(x.view(torch.int16), y.view(torch.int16))  # noqa: E731
    assert same(kp, k0) and same(vp, v0) and same(w, w0) and torch.equal(pos, pos0)


def test_prompt_to_eviction_and_on():
    """As a serving program uses them: prompts in, weights of their keys, eviction, then single tokens against what is left."""
    dt, code = DT["bf16"]
    n, Hq, Hkv, D, page, budget, recent = [600, 90, 333], 8, 2, 128, 32, 128, 16
    scale, B, off = D ** -0.5, 3, _off([600, 90, 333])
    x = _normal(0, off[-1], Hq + 2 * Hkv, D, dtype=dt)
    x[:, :Hq] *= 2.0
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pages, most, table, kp, vp = _pool(n, [4] * B, page, Hkv, D, dt, 1)
    S = pages * page
    w = torch.zeros(Hkv, S, device="cuda")
    pos = torch.zeros(Hkv, S, dtype=torch.int32, device="cuda")
    out, lse, _ = run_prompt(q, k, v, off, code, scale)
    append(k, v, None, off, kp, vp, page, table, [0] * B, w, pos)
    assert weigh(q, code, lse, off, kp, page, table, [0] * B, scale, w).tolist() == [0] * B
    # every row's weights sum to one for each of its heads
    for b in range(B):
        total = w[:, slots(table, b, n[b], page)].double().sum(1)
        assert ((total - n[b] * Hq / Hkv).abs() <= n[b] * Hq / Hkv * 1e-4).all()
    new, _ = evict(kp, vp, page, table, n, n, budget, recent, w, pos)
    assert new == [128, 90, 128]
    for step in range(3):
        ctx = [m + step for m in new]
        one = _normal(50 + step, B, Hq + 2 * Hkv, D, dtype=dt)
        st = append(one[:, Hq:Hq + Hkv], one[:, Hq + Hkv:], _i32([a + step for a in n]), [0, 1, 2, 3], kp, vp, page, table, ctx, w, pos)
        assert st.tolist() == [0] * B
        out, lse, st = run_paged(one[:, :Hq], code, [0, 1, 2, 3], None, kp, vp, page, table, ctx, scale)
        assert st.tolist() == [0] * B
        for b in range(B):
            at = slots(table, b, ctx[b] + 1, page)
            for h in range(Hkv):  # each head has its own tokens: the original rows of their positions
                p = pos[h, at].long()
                old = p < n[b]
                assert torch.equal(kp.view(S, Hkv, D)[at][old, h], k[off[b] + p[old], h])
                assert torch.equal(vp.view(S, Hkv, D)[at][old, h], v[off[b] + p[old], h])
                assert int((p >= n[b] - recent).sum()) >= recent if n[b] > budget else True
            K, V = kp.view(S, Hkv, D)[at], vp.view(S, Hkv, D)[at]
            o, z, o_tol, z_tol = attention(one[b:b + 1, :Hq], K, V, causal_mask(1, ctx[b]), scale)
            check(out[b:b + 1], o, o_tol, "out")
            check(lse[b:b + 1], z, z_tol, "lse")
        assert weigh(one[:, :Hq], code, lse, [0, 1, 2, 3], kp, page, table, ctx, scale, w).tolist() == [0] * B


@pytest.mark.parametrize("n,ctx,D,t", [([64, 90, 33], [20000, 15001, 9000], 64, "f16"), ([50, 1, 70, 200], [12000, 9000, 14000, 100], 128, "bf16")])
def test_weights_of_many_segments(n, ctx, D, t):
    """Far more segments than CTAs, of one, two and more Q tiles."""
    test_weights(n, ctx, 32, 8, D, t, 64)


def test_requests_share_a_prefix():
    """Three requests read one prefix's pages; what they append is their own, and the prefix gains all their weight."""
    page, P, Hq, Hkv, D, t = 16, 320, 8, 2, 128, "bf16"
    dt, code = DT[t]
    n, ctx, scale = [1, 40, 3], [P, P, P + 5], D ** -0.5
    pages, most, table, kp, vp = _pool(n, ctx, page, Hkv, D, dt, 3)
    table[1:, :P // page] = table[0, :P // page]
    S, off = pages * page, _off(n)
    q, k, v = _normal(1, off[-1], Hq, D, dtype=dt), _normal(2, S, Hkv, D, dtype=dt), _normal(3, S, Hkv, D, dtype=dt)
    kp.view(S, Hkv, D).copy_(k)
    vp.view(S, Hkv, D).copy_(v)
    out, lse, status = run_paged(q, code, off, None, kp, vp, page, table, ctx, scale)
    w = torch.zeros(Hkv, S, device="cuda")
    want, tol = torch.zeros(Hkv, S, dtype=torch.float64, device="cuda"), torch.zeros(Hkv, S, dtype=torch.float64, device="cuda")
    for b in range(3):
        a, e, see = off[b], off[b + 1], causal_mask(n[b], ctx[b])
        at = slots(table, b, ctx[b] + n[b], page)
        o, z, o_tol, z_tol = attention(q[a:e], k[at], v[at], see, scale)
        check(out[a:e], o, o_tol, "out")
        check(lse[a:e], z, z_tol, "lse")
        got, t_b = ref_weights(q[a:e], k[at], lse[a:e], see, scale)
        want[:, at] += got
        tol[:, at] += t_b + 2.0 ** -23 * want[:, at]  # one more addition for each request
    assert status.tolist() == [0] * 3
    assert weigh(q, code, lse, off, kp, page, table, ctx, scale, w).tolist() == [0] * 3
    check(w, want, tol, "weights")


@pytest.mark.parametrize("B", [33, 70, 1100])
def test_weights_of_many_requests(B):
    test_weights([i % 3 for i in range(B)], [i * 7 % 40 for i in range(B)], 2, 1, 64, "f16", 8)
