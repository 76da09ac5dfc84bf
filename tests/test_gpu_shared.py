"""The calls together, as a program makes them: rotary positions, the append, attention, branches that share their prompt's pages, a
pool closed up; and the decoding loop over caches in 8 bits and with rotary positions.

The loop must emit the target's greedy tokens (tau = 0) where the cache is in 16 bits: each is the argmax of dense attention in fp32,
or within LOGIT_EPS of it.  The rotary turns add what a rounding to bf16 the other way costs where fp32 and fp64 fall on two sides of
a tie, one value in thousands: within what the outputs' own rounding needs."""
import math

import numpy as np
import pytest
import torch

import coded_ref as cr
from paged_ref import attention, causal_mask, check, tree_mask
from paper_2511_01282_gb300 import respec as rs
from paper_2511_01282_gb300.rotary import Rotary
from paper_2511_01282_gb300.shared import SharedCache

pytestmark = pytest.mark.gpu
LOGIT_EPS = 0.1


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def turned(rot, x, pos):
    """x at the positions, in 64 bits; what fp32 and the rounding of the result may be off by: an angle 2^-24 of half a turn, and
    functions and products of fp32 (2^-22), of the pair's length, and half a step."""
    a = (pos.cpu().double()[:, None] * rot.freq).cuda()[:, None]
    lo, hi = x.double().chunk(2, -1)
    want = torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)
    size = torch.cat([(lo * lo + hi * hi).sqrt()] * 2, -1)
    tiny = torch.finfo(x.dtype).tiny
    return want, size * (math.pi * 2.0 ** -24 + 2.0 ** -21) + (want.abs() + tiny) * torch.finfo(x.dtype).eps / 2


def grid(dt, most):
    """What rounding to the grids of 2^-9 x 2^e may sum up to, for values of at most `most`: half a step at every growth of a block's
    exponent, so less than a step of the last one, and again after the values were appended anew."""
    return 2 * 2.0 ** -9 * 2.0 ** cr.exponent([float(most)], dt)


class Program:
    """Requests over a SharedCache; every request's keys and values beside it, as the cache was given them."""

    def __init__(self, cache, Hq, layout="half"):
        self.c, self.Hq = cache, Hq
        self.rot = Rotary(cache.D, layout=layout)
        self.k, self.v = ([torch.zeros(0, cache.Hkv, cache.D, dtype=cache.dtype, device="cuda") for _ in range(cache.B)] for _ in range(2))
        self.seed, self.most = 0, [0.0, 0.0]

    def step(self, counts, parents=None, max_new=None, checked=True):
        c, T = self.c, sum(counts)
        off = [0]
        for n in counts:
            off.append(off[-1] + n)
        self.seed += 1
        g = torch.Generator().manual_seed(self.seed)
        x = torch.randn(T, self.Hq + 2 * c.Hkv, c.D, generator=g).to(c.dtype).cuda()
        q, k, v = x[:, :self.Hq], x[:, self.Hq:self.Hq + c.Hkv], x[:, self.Hq + c.Hkv:]
        depth = [tree_depths(parents, counts, off, b, i) for b, n in enumerate(counts) for i in range(n)]
        pos = i32([c.seen[b] + depth[off[b] + i] for b, n in enumerate(counts) for i in range(n)])
        want = [turned(self.rot, t, pos) for t in (q, k)]
        self.rot(q, k, pos, out=(q, k))
        for got, (w, tol) in zip((q, k), want):
            assert bool(((got.double() - w).abs() <= tol).all())
        self.most = [max(m, float(t.abs().max())) for m, t in zip(self.most, (k, v))]
        c.reserve(counts)
        c.append(k, v, i32(off))
        tree = None if parents is None else i32(parents)
        out, lse = c.attend(q, i32(off), c.D ** -0.5, tree, max_new)
        if checked:
            if c.bits == 8:
                pool = [(cr.values(codes, e).cuda().view(-1, c.Hkv, c.D), e.repeat_interleave(16, 1).view(-1, c.Hkv))
                        for codes, e in ((c.k, c.k_exps), (c.v, c.v_exps))]
            for b, n in enumerate(counts):
                if not n:
                    continue
                m = c.lengths[b] + n
                at = c.rows(b, torch.arange(m, device="cuda"))
                see = causal_mask(n, c.lengths[b]) if parents is None else torch.cat(
                    [torch.ones(n, c.lengths[b], dtype=torch.bool), tree_mask(parents[off[b]:off[b + 1]])], 1)
                mine = torch.cat([self.k[b], k[off[b]:off[b + 1]]]), torch.cat([self.v[b], v[off[b]:off[b + 1]]])
                if c.bits == 8:
                    both = [(val[at], e[at]) for val, e in pool]
                    for (val, e), true, most in zip(both, mine, self.most):  # e4m3's half step
                        off_by = true.double().abs() * 2.0 ** -4 + grid(c.dtype, most)
                        assert bool(((val - true.double()).abs() <= off_by).all())
                    ref = cr.coded_attention(q[off[b]:off[b + 1]], both[0][0], both[1][0], both[1][1], see, c.D ** -0.5)
                else:
                    assert torch.equal(c.values(at)[0], mine[0]) and torch.equal(c.values(at)[1], mine[1])
                    ref = attention(q[off[b]:off[b + 1]], *mine, see, c.D ** -0.5)
                check(out[off[b]:off[b + 1]], ref[0], ref[2], "out of request %d" % b)
                check(lse[off[b]:off[b + 1]], ref[1], ref[3], "lse of request %d" % b)
        return k, v, off

    def commit(self, new, keep=None):
        k, v, off = new
        counts = []
        for b in range(self.c.B):
            at = list(range(off[b + 1] - off[b])) if keep is None else keep[b]
            if keep is not None:
                self.c.keep(b, at)
            self.k[b] = torch.cat([self.k[b], k[off[b]:off[b + 1]][at]])
            self.v[b] = torch.cat([self.v[b], v[off[b]:off[b + 1]][at]])
            counts.append(len(at))
        self.c.advance(counts)

    def fork(self, src, dsts, n=None):
        self.c.fork(src, dsts, n)
        for b in dsts:
            self.k[b], self.v[b] = self.k[src][:self.c.lengths[b]], self.v[src][:self.c.lengths[b]]

    def free(self, b):
        self.c.free(b)
        self.k[b], self.v[b] = self.k[b][:0], self.v[b][:0]


def tree_depths(parents, counts, off, b, i):
    if parents is None:
        return i
    d = 0
    while parents[off[b] + i] >= 0:
        i, d = parents[off[b] + i], d + 1
    return d


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits,Hq,Hkv,D,page", [(8, 8, 2, 128, 64), (8, 4, 4, 64, 16), (16, 8, 2, 64, 16), (16, 4, 1, 128, 128)])
def test_a_program_of_prompts_branches_trees_and_tokens(dt, bits, Hq, Hkv, D, page):
    p = Program(SharedCache(5, 700, page, Hkv, D, 3200 // page, dtype=dt, bits=bits), Hq, layout="half")
    c = p.c
    p.commit(p.step([300, 37, 0, 0, 0]))
    p.commit(p.step([45, 200, 0, 0, 0]))  # the prompts' next pieces
    p.fork(0, [2, 3])
    p.fork(1, [4], 100)
    used = c.n_pages - c.free_pages
    for _ in range(20):  # branches of one prompt, a token each
        p.commit(p.step([1] * 5, max_new=1))
    assert c.lengths == [365, 257, 365, 365, 120] and c.n_pages - c.free_pages <= used + 5 * -(-20 // page) + 5
    tree = [-1, 0, 0, 1, 1, 2, 3]  # trees behind two of them, an accepted path of each
    new = p.step([7, 0, 7, 0, 0], parents=tree * 2, max_new=7)
    p.commit(new, keep=[[0, 1, 4], [], [0, 2, 5], [], []])
    p.free(0)
    p.free(1)
    at = c.k.data_ptr()
    c.resize(c.n_pages - c.free_pages + 2 * 3)
    assert c.k.data_ptr() != at and max(x for h in c.held for x in h) < c.n_pages - 6
    for n in ([0, 0, 3, 2, 1], [0, 0, 1, 1, 1]):
        p.commit(p.step(n, max_new=3))
    p.fork(2, [0], 300)
    p.commit(p.step([4, 0, 1, 0, 2], max_new=4))
    for b in (0, 2, 3, 4):
        p.free(b)
    assert c.free_pages == c.n_pages and c.compact() == 0
    c.check()


def test_a_captured_step_goes_on_over_pages_that_are_reserved_between():
    """rotary, append and attention as one graph over a batch of branches; pages, lengths and positions change between its replays."""
    dt, Hq, Hkv, D, B = torch.bfloat16, 8, 2, 128, 3
    c = SharedCache(B, 400, 32, Hkv, D, 40, dtype=dt, bits=8)
    p = Program(c, Hq)
    p.commit(p.step([90, 0, 0]))
    p.fork(0, [1, 2])
    x = torch.zeros(B, Hq + 2 * Hkv, D, dtype=dt, device="cuda")
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q2, k2 = torch.empty(B, Hq, D, dtype=dt, device="cuda"), torch.empty(B, Hkv, D, dtype=dt, device="cuda")
    off, pos = i32([0, 1, 2, 3]), c.next

    def run():
        p.rot(q, k, pos, out=(q2, k2))
        c.append(k2, v, off)
        return c.attend(q2, off, D ** -0.5, max_new=1)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.reserve([1] * B)
        run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = run()
    for i in range(40):
        c.reserve([1] * B)
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(900 + i)).to(dt))
        graph.replay()
        got = out.clone(), lse.clone(), [a.clone() for a in c._arrays()]
        eager = run()  # the same again: the token's codes are written over by themselves
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1]) and all(torch.equal(a, b) for a, b in zip(got[2], c._arrays()))
        c.advance([1] * B)
    c.check()
    assert c.lengths == [130] * B and len({tuple(h) for h in c.held}) == B


def test_branches_of_a_tracked_cache_are_evicted_apart():
    c = SharedCache(3, 300, 16, 2, 64, 60, track_weights=True)
    p = Program(c, 4)
    new = p.step([150, 0, 0])
    p.commit(new)
    c.weights.uniform_()
    p.fork(0, [1, 2])
    rows = [c.rows(b, torch.arange(150, device="cuda")) for b in range(3)]
    for x in (c.weights, c.positions):
        assert torch.equal(x[:, rows[0]], x[:, rows[1]]) and torch.equal(x[:, rows[0]], x[:, rows[2]])
    c.weights[:, rows[1]] = 1.0 - c.weights[:, rows[1]]
    first = [x[:, rows[2]].clone() for x in (c.weights, c.positions)] + [a.clone() for a in c.values(rows[2])]
    c.evict([150, 150, 150], 150, 10)  # nothing to do
    c.free(2)
    c.evict([150, 150, 0], 100, 10)
    assert c.lengths == [100, 100, 0]
    kept = [set(c.positions[0, c.rows(b, torch.arange(100, device="cuda"))].tolist()) for b in (0, 1)]
    assert kept[0] != kept[1] and all(set(range(140, 150)) <= x for x in kept)
    c.trim(0)
    c.trim(1)
    assert [len(h) for h in c.held] == [7, 7, 0]
    before = [(c.weights[:, r].clone(), c.positions[:, r].clone(), *c.values(r)) for r in (c.rows(b, torch.arange(100, device="cuda")) for b in (0, 1))]
    c.resize(14)
    after = [(c.weights[:, r].clone(), c.positions[:, r].clone(), *c.values(r)) for r in (c.rows(b, torch.arange(100, device="cuda")) for b in (0, 1))]
    assert all(torch.equal(a, b) for x, y in zip(before, after) for a, b in zip(x, y))
    assert len(first) == 4
    c.check()


# ------------------------------------------------------------------ the loop
def _loop(n, prompt_len=300, seed=0, rotary=False, **kw):
    from paper_2511_01282_gb300.e2e import SpecLoop, TinyLM, make_prompt
    target = TinyLM(seed=seed, rotary=rotary)
    draft = TinyLM(seed=seed + 1, base=target, noise=0.1, rotary=rotary)
    prompt = make_prompt(target.V, prompt_len, seed=seed + 2)
    loop = SpecLoop(target, draft, prompt, rs.params(tau=0.0, span_len=8), **kw)
    return target, prompt, loop, loop.generate(n)


@pytest.mark.parametrize("kw", [dict(cache="flat"), dict(cache="paged", page_size=16)])
def test_the_loop_with_rotary_positions_emits_the_targets_greedy_tokens(kw):
    target, prompt, loop, got = _loop(64, rotary=True, **kw)
    seq = torch.as_tensor(np.concatenate([prompt, got]), dtype=torch.int64, device=target.device)
    L = target.dense_logits(seq)[len(prompt) - 1:-1]
    gap = L.max(-1).values - L.gather(1, torch.as_tensor(got, device=target.device)[:, None]).squeeze(1)
    assert float(gap.max()) <= LOGIT_EPS and int((gap > 0).sum()) <= 3
    assert loop.stats["steps"] < 64


@pytest.mark.parametrize("rotary", [False, True])
def test_the_loop_in_8_bits_keeps_every_committed_token(rotary):
    """The first layer's keys and values depend on the token and its position alone.  They are bf16 numbers of a product that another
    batch may round otherwise (a step of 2^-7 at most, and 2^-18 of a head's size before the rounding), in e4m3 (2^-4)."""
    target, prompt, loop, got = _loop(60, rotary=rotary, cache="paged", page_size=16, bits=8)
    assert len(got) == 60 and loop.tc["S"] == loop.tc["seen"] == loop.n - 1
    layer, n = loop.tc["layers"][0], loop.n - 1
    assert layer.lengths == [n]
    tokens = loop.buf[:n].long()
    pos = torch.arange(n, dtype=torch.int32, device="cuda") if rotary else None
    q, k, v = target._qkv(target.p["emb"][tokens], 0, pos)
    at = layer.rows(0, torch.arange(n, device="cuda"))
    words = [x.abs().max() * 2 ** 0.5 for x in target._qkv(target.p["emb"], 0, None)[1:]]  # no tree holds a larger one, turned
    for have, want, most in zip(layer.values(at), (k, v), words):
        want = want.double()
        near = 2.0 ** -18 * want.abs().amax(-1, keepdim=True)
        tol = want.abs() * (2.0 ** -7 + 2.0 ** -4 * (1 + 2.0 ** -7)) + near * 1.1 + grid(torch.bfloat16, most)
        assert bool(((have.double() - want).abs() <= tol).all())
