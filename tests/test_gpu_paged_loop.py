"""The decoding loop with paged caches, and PagedCache on more than one request.

Without a budget the loop must emit the target's greedy tokens (tau = 0).  Each token is checked against dense attention in
fp32: the argmax, or within LOGIT_EPS of it.  Beside P the paged call rounds its outputs to bf16, one more relative 2^-9 per
attention output, so the flat loop's 0.05 doubles."""
import numpy as np
import pytest
import torch

from paged_ref import attention, causal_mask, check
from paper_2511_01282_gb300 import respec as rs

pytestmark = pytest.mark.gpu
LOGIT_EPS = 0.1


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _loop(n, prompt_len=300, seed=0, **kw):
    from paper_2511_01282_gb300.e2e import SpecLoop, TinyLM, make_prompt
    target = TinyLM(seed=seed)
    draft = TinyLM(seed=seed + 1, base=target, noise=0.1)
    prompt = make_prompt(target.V, prompt_len, seed=seed + 2)
    loop = SpecLoop(target, draft, prompt, rs.params(tau=0.0, span_len=8), cache="paged", **kw)
    return target, prompt, loop, loop.generate(n)


@pytest.mark.parametrize("page_size", [16, 128])
def test_the_paged_loop_emits_the_targets_greedy_tokens(page_size):
    target, prompt, loop, got = _loop(96, page_size=page_size)
    seq = torch.as_tensor(np.concatenate([prompt, got]), dtype=torch.int64, device=target.device)
    L = target.dense_logits(seq)[len(prompt) - 1:-1]
    gap = L.max(-1).values - L.gather(1, torch.as_tensor(got, device=target.device)[:, None]).squeeze(1)
    assert float(gap.max()) <= LOGIT_EPS and int((gap > 0).sum()) <= 3
    assert loop.stats["steps"] < 96 and loop.tc["S"] == loop.tc["seen"] == loop.n - 1


def test_a_prompt_of_one_token():
    target, prompt, loop, got = _loop(8, prompt_len=1)
    assert len(got) == 8 and loop.n >= 9


def test_the_budgeted_loop_keeps_its_budget():
    budget, recent = 96, 32
    target, prompt, loop, got = _loop(60, budget=budget, recent=recent)
    assert len(got) == 60
    for cache in (loop.tc, loop.dc):
        assert cache["S"] <= budget and cache["seen"] == loop.n - 1
        for layer in cache["layers"]:
            n = layer.lengths[0]
            at = layer.rows(0, torch.arange(n, device="cuda"))
            pos = layer.positions[:, at]
            for h in range(layer.Hkv):  # every token once, all recent ones among them
                p = sorted(pos[h].tolist())
                assert len(set(p)) == n and p[-1] < cache["seen"]
                assert p[-recent:] == list(range(cache["seen"] - recent, cache["seen"]))
            w = layer.weights[:, at]
            assert bool((w >= 0).all()) and bool(torch.isfinite(w).all())


def test_paged_cache_of_several_requests():
    from paper_2511_01282_gb300.paged import PagedCache, prompt_attention
    dt, Hq, Hkv, D = torch.float16, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    n = [40, 7]
    off = torch.tensor([0, 40, 47], dtype=torch.int32, device="cuda")
    x = torch.randn(47, Hq + 2 * Hkv, D, generator=g, device="cuda").to(dt)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    out, lse, status, _ = prompt_attention(q, k, v, off, 0.125)
    c = PagedCache(2, 64, 16, Hkv, D, dtype=dt, track_weights=True)
    c.append(k, v, off)
    again, lse2 = c.attend(q, off, 0.125)  # the whole prompt as a chunk
    assert status.tolist() == [0, 0] and c.status.tolist() == [0, 0]
    for b in range(2):
        a, e = int(off[b]), int(off[b + 1])
        o, z, o_tol, z_tol = attention(q[a:e], k[a:e], v[a:e], causal_mask(n[b], 0), 0.125)
        for got, l in ((out, lse), (again, lse2)):
            check(got[a:e], o, o_tol, "out")
            check(l[a:e], z, z_tol, "lse")
    c.weigh(q, lse, off, 0.125)
    c.advance(n)
    c.evict([40, 7], 10, 4)
    assert c.lengths == [10, 7] and c.length.tolist() == [10, 7]
    pos = c.positions[:, c.rows(0, torch.arange(10, device="cuda"))]
    assert all(set(range(36, 40)) <= set(p) for p in pos.tolist())


def test_captured_cache_calls_keep_their_scratch():
    """A graph of a cache's calls is replayed after larger eager calls of the same cache, their memory in use again."""
    from paper_2511_01282_gb300.paged import PagedCache
    dt, Hq, Hkv, D = torch.bfloat16, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = lambda n: torch.randn(n, Hq + 2 * Hkv, D, generator=g, device="cuda").to(dt)  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = PagedCache(2, 1024, 16, Hkv, D, dtype=dt, track_weights=True)
    first, off = rows(600), i32(0, 400, 600)
    c.append(first[:, Hq:Hq + Hkv], first[:, Hq + Hkv:], off)
    c.advance([400, 200])
    x, small = rows(2), i32(0, 1, 2)

    def step():
        c.append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], small)
        out, lse = c.attend(x[:, :Hq], small, 0.09)
        c.weigh(x[:, :Hq], lse, small, 0.09)
        return out, lse

    step()
    weights = c.weights.clone()
    c.weights.zero_()
    want = [t.clone() for t in step()] + [c.weights.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    big, big_off = rows(700), i32(0, 500, 700)
    c.append(big[:, Hq:Hq + Hkv], big[:, Hq + Hkv:], big_off)
    c.attend(big[:, :Hq], big_off, 0.09)
    filler = [torch.full((1 << n,), 77, dtype=torch.uint8, device="cuda") for n in range(12, 27)]
    c.weights.copy_(0 * weights)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(c.weights, want[2])
    assert all(bool((f == 77).all()) for f in filler)
