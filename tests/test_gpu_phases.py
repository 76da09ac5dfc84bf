"""Attention worked off in groups of KV heads (more keys than L2 holds, read by several pairs of row tiles): chunks and trees over
pages, both head sizes, numbers of heads that the groups do not divide.  Rows of every head against the formula."""
import pytest
import torch

from paged_ref import attention, check, slots, tree_mask
from paper_2511_01282_gb300 import respec as rs
from test_gpu_prompt_paged import DT, _i32, _normal, _off, _pool, _trees, run_paged, run_prompt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _groups(n, ctx, tree, Hq, Hkv, D):
    """How many groups the plan makes of the heads, by its rule (about, for prompts): keys of all requests against L2, key tiles
    of a share."""
    p = torch.cuda.get_device_properties(0)
    sms, l2, tq = min(p.multi_processor_count, 512), p.L2_cache_size, 128 // (Hq // Hkv)
    tiles = sum(-(-a // (2 * tq)) * (c + (a if tree else a // 2)) // 128 for a, c in zip(n, ctx))
    used = 4.0 * Hkv * D * sum(a + c for a, c in zip(n, ctx))
    g = 1
    while g < 4 and 2 * g <= Hkv and used > 1.5 * l2 and used > 0.5 * l2 * g and tiles * Hkv // (sms * 2 * g) >= 200:
        g *= 2
    return g


@pytest.mark.parametrize("n,ctx,Hq,Hkv,D,t,page,tree,groups", [
    ([700, 90], [150000, 60000], 48, 6, 64, "bf16", 64, False, 4),    # groups of one and of two heads
    ([256, 200], [230000, 170000], 48, 6, 64, "f16", 16, True, 4),
    ([1500], [100000], 40, 5, 128, "bf16", 128, False, 4),
    ([600], [160000], 24, 3, 128, "f16", 8, False, 2),
])
def test_pages(n, ctx, Hq, Hkv, D, t, page, tree, groups):
    assert _groups(n, ctx, tree, Hq, Hkv, D) == groups
    dt, code = DT[t]
    pages, most, table, kp, vp = _pool(n, ctx, page, Hkv, D, dt, 3)
    kp, vp = _normal(7, *kp.shape, dtype=dt), _normal(8, *vp.shape, dtype=dt)
    off = _off(n)
    q = _normal(1, off[-1], Hq, D, dtype=dt)
    par = _trees(n, 7) if tree else None
    out, lse, status = run_paged(q, code, off, _i32(sum(par, [])) if tree else None, kp, vp, page, table, ctx, D ** -0.5)
    assert status.tolist() == [0] * len(n)
    for b in range(len(n)):
        at = slots(table, b, ctx[b] + n[b], page)
        K, V = kp.view(-1, Hkv, D)[at], vp.view(-1, Hkv, D)[at]
        for i in (0, n[b] // 2, n[b] - 1):
            if tree:
                see = torch.cat([torch.ones(ctx[b], dtype=torch.bool), tree_mask(par[b])[i]])[None]
            else:
                see = torch.arange(ctx[b] + n[b])[None] <= ctx[b] + i
            r = off[b] + i
            o, z, o_tol, z_tol = attention(q[r:r + 1], K, V, see, D ** -0.5)
            check(out[r:r + 1], o, o_tol, "row %d of request %d" % (i, b))
            check(lse[r:r + 1], z, z_tol, "lse of row %d of request %d" % (i, b))
    again = run_paged(q, code, off, _i32(sum(par, [])) if tree else None, kp, vp, page, table, ctx, D ** -0.5)
    assert torch.equal(again[0].view(torch.int16), out.view(torch.int16)) and torch.equal(again[1], lse)


def test_a_prompt_of_heads_that_the_groups_do_not_divide():
    T, Hq, Hkv, D = 90000, 20, 5, 128
    assert _groups([T], [0], False, Hq, Hkv, D) == 4
    q, k, v = (_normal(s, T, h, D, dtype=torch.bfloat16) for s, h in ((0, Hq), (1, Hkv), (2, Hkv)))
    out, lse, status = run_prompt(q, k, v, [0, T], rs.RS_BF16, 0.09)
    assert status.tolist() == [0]
    for i in (0, 63, 64, 20000, T - 1):
        o, z, o_tol, z_tol = attention(q[i:i + 1], k[:i + 1], v[:i + 1], torch.ones(1, i + 1, dtype=torch.bool), 0.09)
        check(out[i:i + 1], o, o_tol, "row %d" % i)
        check(lse[i:i + 1], z, z_tol, "lse of row %d" % i)
