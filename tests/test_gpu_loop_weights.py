"""The weights and choices that the budgeted decoding loop lives by, against the formulas."""
import pytest
import torch

from paged_ref import causal_mask, check, evict_order, weights as ref_weights
from test_gpu_loop_status import _loop

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def test_every_row_of_the_loop_gives_its_whole_weight():
    """Before the first eviction each head's weights sum to one for every token and query head."""
    loop = _loop(budget=600, recent=32)
    loop.generate(60)
    for cache in (loop.tc, loop.dc):
        assert cache["S"] == cache["seen"] == loop.n - 1
        for layer in cache["layers"]:
            n = layer.lengths[0]
            total = layer.weights[:, layer.rows(0, torch.arange(n, device="cuda"))].double().sum(1)
            want = n * 4 / 2
            # lse and its exponentials are off by 2^-19 or so of |score| < 32 each, and n fp32 additions to a sum
            assert ((total - want).abs() <= want * 1e-4).all()


def test_the_loop_weighs_and_evicts_by_the_formula(monkeypatch):
    """Every commit's weights against the formula on the rows and keys of that layer, every eviction against the order."""
    from paper_2511_01282_gb300.paged import PagedCache
    real_weigh, real_evict, seen = PagedCache.weigh, PagedCache.evict, dict(weigh=0, evict=0)

    def weigh(self, q, lse, new_off, scale):
        n, ctx = q.shape[0], self.lengths[0]
        at = self.rows(0, torch.arange(ctx + n, device="cuda"))
        before = self.weights[:, at].double()
        K = self.k.view(-1, self.Hkv, self.D)[at]
        assert bool((before[:, ctx:] == 0).all())  # new tokens begin without weight
        real_weigh(self, q, lse, new_off, scale)
        got, tol = ref_weights(q, K, lse, causal_mask(n, ctx), scale)
        check(self.weights[:, at], before + got, tol + 2.0 ** -23 * (before + got), "weights")
        assert ((got.sum(1) - n * q.shape[1] / self.Hkv).abs() < 1e-2 * n).all()  # q, lse and the keys belong together
        seen["weigh"] += 1

    def evict(self, next_pos, budget, recent):
        n = self.lengths[0]
        at = self.rows(0, torch.arange(n, device="cuda"))
        w, pos = self.weights[:, at].tolist(), self.positions[:, at].tolist()
        assert all(sorted(p)[-1] == next_pos[0] - 1 for p in pos)
        real_evict(self, next_pos, budget, recent)
        for h in range(self.Hkv):
            want = list(pos[h][:budget])
            for src, dst in evict_order(w[h], pos[h], next_pos[0], recent, budget):
                want[dst] = pos[h][src]
            assert self.positions[h, at[:budget]].tolist() == want
        seen["evict"] += 1

    monkeypatch.setattr(PagedCache, "weigh", weigh)
    monkeypatch.setattr(PagedCache, "evict", evict)
    loop = _loop(budget=96, recent=32)
    loop.generate(40)
    steps = loop.stats["steps"]
    assert seen["weigh"] == 4 * (steps + 1) and 4 * steps <= seen["evict"] <= 4 * (steps + 1)  # two models of two layers
