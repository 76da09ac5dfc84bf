"""Values that a row does not see: NaN and infinity in V stay with the rows that see them, but for those that share both a row
tile and a tile of 128 keys with such a row (a hidden key there has weight 0, and 0 times NaN is NaN)."""
import pytest
import torch

from paged_ref import attention, causal_mask, check, slots
from test_gpu_prompt_paged import DT, _normal, _off, _pool, run_paged, run_prompt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _out_of_reach(n, ctx, G, j):
    """[n] rows whose row tile (128 / G tokens) ends in an earlier key tile than token j's."""
    tq = 128 // G
    last = torch.tensor([min(n, (i // tq + 1) * tq) - 1 for i in range(n)])
    return (ctx + last) // 128 < (ctx + j) // 128


def _check_rows(q, k, v, out, lse, n, ctx, j, scale):
    """Rows out of reach of token j are the formula's; those that see it are not finite; every lse is the formula's."""
    G = q.shape[1] // k.shape[1]
    clean = v.clone()
    clean[ctx + j] = 0.0
    o, z, o_tol, z_tol = attention(q, k, clean, causal_mask(n, ctx), scale)
    far = _out_of_reach(n, ctx, G, j).to(out.device)
    check(out[far], o[far], o_tol[far], "rows that do not see token %d" % j)
    assert not bool(torch.isfinite(out[j:]).any())
    check(lse, z, z_tol, "lse")
    return int(far.sum())


@pytest.mark.parametrize("n,Hq,Hkv,D,t,j,value", [
    (256, 2, 2, 64, "bf16", 200, "nan"),     # one pair of row tiles
    (256, 1, 1, 128, "f16", 255, "inf"),
    (300, 6, 2, 128, "bf16", 130, "nan"),    # 42 tokens to a row tile
    (300, 6, 2, 64, "f16", 290, "-inf"),
    (1400, 5, 5, 128, "bf16", 1300, "nan"),
    (1400, 5, 5, 64, "f16", 1025, "nan"),
])
def test_prompts(n, Hq, Hkv, D, t, j, value):
    dt, code = DT[t]
    off = _off([70, n])
    q, k, v = (_normal(s, off[-1], h, D, dtype=dt) for s, h in ((0, Hq), (1, Hkv), (2, Hkv)))
    v[70 + j] = float(value)
    out, lse, status = run_prompt(q, k, v, off, code, D ** -0.5)
    assert status.tolist() == [0, 0]
    assert bool(torch.isfinite(out[:70]).all())
    assert _check_rows(q[70:], k[70:], v[70:], out[70:], lse[70:], n, 0, j, D ** -0.5) >= min(j // 128 * 128, 84)


@pytest.mark.parametrize("Hq,Hkv,D,t", [(1, 1, 64, "bf16"), (2, 2, 128, "f16"), (6, 2, 128, "bf16"), (3, 1, 64, "f16")])
def test_chunks_behind_every_length(Hq, Hkv, D, t):
    """Cached tokens of many numbers: the shares' ends cut the segments everywhere, also where a piece holds only keys that
    the first row tile does not see."""
    dt, code = DT[t]
    n, page = 2 * (128 // (Hq // Hkv)), 32
    q = _normal(0, n, Hq, D, dtype=dt)
    for ctx in list(range(0, 1200, 57)) + [3000, 5003, 9999]:
        pages, most, table, kp, vp = _pool([n], [ctx], page, Hkv, D, dt, 5)
        at = slots(table, 0, ctx + n, page)
        k, v = _normal(1, ctx + n, Hkv, D, dtype=dt), _normal(2, ctx + n, Hkv, D, dtype=dt)
        j = n - 1
        v[ctx + j] = float("nan")
        kp.view(-1, Hkv, D)[at] = k
        vp.view(-1, Hkv, D)[at] = v
        out, lse, status = run_paged(q, code, [0, n], None, kp, vp, page, table, [ctx], D ** -0.5)
        assert status.tolist() == [0]
        _check_rows(q, k, v, out, lse, n, ctx, j, D ** -0.5)


@pytest.mark.parametrize("D,t", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("n", [40, 700])
def test_rows_without_weight_give_zeros_whatever_v_holds(n, D, t):
    dt, code = DT[t]
    q, k, v = (_normal(s, n, 2, D, dtype=dt) for s in (0, 1, 2))
    q = q.abs() + 0.1
    k[:] = float("-inf")
    v[n // 2:] = float("nan")
    out, lse, status = run_prompt(q, k, v, [0, n], code, D ** -0.5)
    assert status.tolist() == [0] and bool((out == 0).all()) and bool(torch.isneginf(lse).all())
