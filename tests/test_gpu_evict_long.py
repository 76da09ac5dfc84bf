"""rs_paged_evict on caches whose keys shared memory does not hold: the selection reads them again in every pass."""
import pytest
import torch

from paged_ref import evict_order, slots
from test_gpu_evict import evict
from test_gpu_prompt_paged import _pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("length,budget,recent,Hkv,page", [
    ([400001], 1500, 100, 1, 256),              # a cluster of eight CTAs holds 393216
    ([400001], 390000, 0, 2, 65536),
    ([50001, 49153, 30, 700], 3000, 64, 20, 64),  # a CTA alone, 49152
])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_long_caches(length, budget, recent, Hkv, page, kind):
    B, D = len(length), 64
    pages, most, table, kp, vp = _pool(length, [0] * B, page, Hkv, D, torch.bfloat16, 8, spare=1)
    S = pages * page
    g = torch.Generator(device="cuda").manual_seed(budget)
    bits = lambda: torch.randint(-32768, 32767, kp.shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)  # noqa: E731
    kp, vp = bits(), bits()
    w = torch.randn(Hkv, S, generator=g, device="cuda")
    if kind == "ties":
        w = (w * 1.5).round()
    pos = torch.stack([torch.randperm(S, generator=g, device="cuda") for _ in range(Hkv)]).int()
    nxt = [S] * B
    k0, v0, w0, pos0 = (x.clone() for x in (kp, vp, w, pos))
    new, status = evict(kp, vp, page, table, length, nxt, budget, recent, w, pos)
    assert new == [min(x, budget) for x in length] and status == [0] * B
    for b in range(B):
        at = slots(table, b, length[b], page)
        if length[b] <= budget:
            continue
        for h in range(Hkv):
            moves = torch.tensor(evict_order(w0[h, at].tolist(), pos0[h, at].tolist(), nxt[b], recent, budget), device="cuda")
            a, d = at[moves[:, 0]], at[moves[:, 1]]
            k0.view(S, Hkv, D)[d, h] = k0.view(S, Hkv, D)[a, h]
            v0.view(S, Hkv, D)[d, h] = v0.view(S, Hkv, D)[a, h]
            w0[h, d], pos0[h, d] = w0[h, a], pos0[h, a]
    same = lambda x, y: torch.equal(x.view(torch.int16), y.view(torch.int16))  # noqa: E731
    assert same(kp, k0) and same(vp, v0) and same(w, w0) and torch.equal(pos, pos0)
