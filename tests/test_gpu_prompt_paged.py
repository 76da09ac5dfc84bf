"""rs_prompt_attn, rs_paged_append and rs_paged_attn against the formulas in 64 bits: types, head layouts, lengths from none to
several key tiles, trees, small pages, strides, values that must not matter."""
import pytest
import torch

from paged_ref import attention, causal_mask, check, slots, tree_mask
from paper_2511_01282_gb300 import respec as rs

pytestmark = pytest.mark.gpu
DT = {"bf16": (torch.bfloat16, rs.RS_BF16), "f16": (torch.float16, rs.RS_F16)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _off(n):
    o = [0]
    for x in n:
        o.append(o[-1] + x)
    return o


def _normal(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _scratch(n):
    return torch.full((max(n, 256),), 0xA5, dtype=torch.uint8, device="cuda")


def run_prompt(q, k, v, off, dtype, scale, tail=0):
    T, Hq, D = q.shape
    Hkv, B = k.shape[1], len(off) - 1
    out = torch.full((T, Hq, D), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    status = torch.full((max(B, 1),), -1, dtype=torch.int32, device="cuda")
    ws = _scratch(rs.rs_prompt_attn_workspace_size(B, T, Hq, Hkv, D))
    rs.rs_prompt_attn(q, q.stride(0), k, k.stride(0), v, v.stride(0), dtype, _i32(off), B, T, Hq, Hkv, D, scale, out, lse, status, ws)
    return out, lse, status


PROMPTS = [
    # lengths, Hq, Hkv, D, type
    ([1], 1, 1, 64, "bf16"),
    ([1, 2, 3], 4, 4, 128, "f16"),
    ([127, 0, 128, 129], 4, 2, 128, "bf16"),
    ([0, 0, 300], 8, 1, 64, "f16"),
    ([255, 256, 257], 3, 1, 128, "bf16"),
    ([33, 700], 14, 2, 64, "bf16"),
    ([1000], 32, 8, 128, "f16"),
    ([5, 1, 411, 64, 0, 90], 40, 40, 64, "f16"),
    ([70], 128, 1, 128, "bf16"),
    ([2100, 31], 6, 2, 128, "bf16"),
]


@pytest.mark.parametrize("n,Hq,Hkv,D,t", PROMPTS)
def test_prompt(n, Hq, Hkv, D, t):
    dt, code = DT[t]
    off = _off(n)
    T, tail = off[-1], 3
    x = _normal(len(n) + D, T + tail, Hq + 2 * Hkv, D, dtype=dt)  # one projection's rows, and some behind the last sequence
    x[:, :Hq] *= 2.0
    x[T:] = float("nan")
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    out, lse, status = run_prompt(q, k, v, off, code, D ** -0.5)
    assert status.tolist() == [0] * len(n)
    assert (out[T:] == 7.0).all() and (lse[T:] == 7.0).all()
    for b in range(len(n)):
        a, e = off[b], off[b + 1]
        if a == e:
            continue
        o, z, o_tol, z_tol = attention(q[a:e], k[a:e], v[a:e], causal_mask(n[b], 0), D ** -0.5)
        check(out[a:e], o, o_tol, "out of sequence %d" % b)
        check(lse[a:e], z, z_tol, "lse of sequence %d" % b)
    again = run_prompt(q, k, v, off, code, D ** -0.5)
    assert torch.equal(again[0][:T].view(torch.int16), out[:T].view(torch.int16)) and torch.equal(again[1][:T], lse[:T])


def _pool(n, ctx, page, Hkv, D, dt, seed, spare=2):
    need = [-(-(a + c) // page) for a, c in zip(n, ctx)]
    pages, most = sum(need) + spare, max(max(need), 1)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table, at = [], 0
    for x in need:
        table.append(order[at:at + x] + [1 << 30] * (most - x))  # entries behind a request's pages are never read
        at += x
    nan = lambda: torch.full((pages, page, Hkv, D), float("nan"), dtype=dt, device="cuda")  # noqa: E731
    return pages, most, _i32(table).view(len(n), most), nan(), nan()


def append(k, v, pos, off, kp, vp, page, table, ctx, weights=None, positions=None):
    B, T, Hkv, D = len(off) - 1, k.shape[0], k.shape[1], k.shape[2]
    status = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    rs.rs_paged_append(k, k.stride(0), v, v.stride(0), pos, _i32(off), B, T, Hkv, D, kp, vp, kp.shape[0], page, table,
                       table.shape[1], _i32(ctx), weights, positions, status)
    return status


def run_paged(q, code, off, parents, kp, vp, page, table, ctx, scale):
    T, Hq, D = q.shape
    B, Hkv = len(off) - 1, kp.shape[2]
    out = torch.full((T, Hq, D), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    status = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ws = _scratch(rs.rs_paged_attn_workspace_size(B, T, Hq, Hkv, D))
    rs.rs_paged_attn(q, q.stride(0), code, _i32(off), parents, B, T, Hq, Hkv, D, kp, vp, kp.shape[0], page, table, table.shape[1],
                     _i32(ctx), scale, out, lse, status, ws)
    return out, lse, status


def _trees(n, seed):
    g = torch.Generator().manual_seed(seed)
    out = []
    for m in n:
        out.append([-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, m)])
    return out


CHUNKS = [
    # new, cached, Hq, Hkv, D, type, page, tree
    ([1], [0], 1, 1, 64, "bf16", 8, False),
    ([1, 1, 1], [0, 127, 128], 8, 2, 128, "f16", 16, False),
    ([1, 0, 1], [5000, 300, 77], 32, 8, 128, "bf16", 64, False),
    ([1] * 20, [37 * i for i in range(20)], 7, 1, 64, "f16", 32, False),
    ([130, 3], [200, 0], 4, 4, 128, "bf16", 128, False),
    ([300, 1, 64], [1000, 2500, 130], 8, 2, 64, "bf16", 8, False),
    ([129], [3000], 6, 2, 128, "f16", 256, False),
    ([1], [20000], 4, 1, 128, "bf16", 16, False),
    ([9, 65], [0, 300], 4, 4, 64, "bf16", 16, True),
    ([256, 1, 40], [90, 128, 1], 8, 2, 128, "f16", 32, True),
    ([65], [4000], 5, 5, 128, "bf16", 128, True),
]


@pytest.mark.parametrize("n,ctx,Hq,Hkv,D,t,page,tree", CHUNKS)
def test_append_then_attend(n, ctx, Hq, Hkv, D, t, page, tree):
    dt, code = DT[t]
    scale = D ** -0.5
    pages, most, table, kp, vp = _pool(n, ctx, page, Hkv, D, dt, 5)
    K = [_normal(100 + b, c + a, Hkv, D, dtype=dt) for b, (a, c) in enumerate(zip(n, ctx))]
    V = [_normal(200 + b, c + a, Hkv, D, dtype=dt) for b, (a, c) in enumerate(zip(n, ctx))]
    S = pages * page
    weights = torch.full((Hkv, S), 3.0, device="cuda")
    positions = torch.full((Hkv, S), -9, dtype=torch.int32, device="cuda")
    # the cached tokens, then the chunk, its rows part of wider ones
    old = _off(ctx)
    st = append(torch.cat([x[:c] for x, c in zip(K, ctx)]), torch.cat([x[:c] for x, c in zip(V, ctx)]), None, old, kp, vp, page, table,
                [0] * len(n), weights, positions)
    assert st.tolist() == [0] * len(n)
    off = _off(n)
    wide = torch.cat([torch.cat([x[c:] for x, c in zip(K, ctx)]), torch.cat([x[c:] for x, c in zip(V, ctx)])], 1)
    pos = _i32([1000 + i for i in range(off[-1])])
    st = append(wide[:, :Hkv], wide[:, Hkv:], pos, off, kp, vp, page, table, ctx, weights, positions)
    assert st.tolist() == [0] * len(n)
    held = torch.zeros(S, dtype=torch.bool, device="cuda")
    for b in range(len(n)):
        at = slots(table, b, ctx[b] + n[b], page)
        held[at] = True
        assert torch.equal(kp.view(S, Hkv, D)[at], K[b]) and torch.equal(vp.view(S, Hkv, D)[at], V[b])
        want = torch.cat([torch.arange(ctx[b]), 1000 + torch.arange(off[b], off[b + 1])]).int().cuda()
        assert (positions[:, at] == want).all() and (weights[:, at] == 0).all()
    assert kp.view(S, Hkv, D)[~held].isnan().all() and vp.view(S, Hkv, D)[~held].isnan().all()
    assert (weights[:, ~held] == 3.0).all() and (positions[:, ~held] == -9).all()

    q = _normal(300, off[-1] + 2, Hq, D, dtype=dt) * 2.0  # two rows behind the last request
    par = _trees(n, 7) if tree else None
    parents = _i32(sum(par, []) + [0, 0]) if tree else None
    out, lse, status = run_paged(q, code, off, parents, kp, vp, page, table, ctx, scale)
    assert status.tolist() == [0] * len(n)
    assert (out[off[-1]:] == 7.0).all() and (lse[off[-1]:] == 7.0).all()
    for b in range(len(n)):
        a, e = off[b], off[b + 1]
        if a == e:
            continue
        see = causal_mask(n[b], ctx[b])
        if tree:
            see = torch.cat([torch.ones(n[b], ctx[b], dtype=torch.bool), tree_mask(par[b])], 1)
        o, z, o_tol, z_tol = attention(q[a:e], K[b], V[b], see, scale)
        check(out[a:e], o, o_tol, "out of request %d" % b)
        check(lse[a:e], z, z_tol, "lse of request %d" % b)


@pytest.mark.parametrize("B,D,t", [(33, 64, "f16"), (70, 128, "bf16"), (1100, 64, "bf16")])
def test_many_requests(B, D, t):
    """More requests than a warp, and than a block, has threads."""
    test_prompt([i * 5 % 7 for i in range(B)], 2, 1, D, t)
    test_append_then_attend([i % 3 for i in range(B)], [i * 7 % 40 for i in range(B)], 2, 1, D, t, 8, False)


def test_many_pairs_of_row_tiles():
    """One prompt of more pairs than a block has threads: 128 heads on one, one token to a row tile."""
    test_prompt([2300], 128, 1, 64, "f16")
