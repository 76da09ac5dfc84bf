"""SharedCache, and PagedCache in 8 bits, on the host: the library's calls are stood in for by their rules on the CPU."""
import random

import pytest
import torch

import coded_ref as cr
from paper_2511_01282_gb300 import respec as rs
from paper_2511_01282_gb300.paged import PagedCache
from paper_2511_01282_gb300.shared import SharedCache


def _arrays(args):
    """Arrays of rs_pages_copy and rs_pages_compact with a page to a row."""
    k, v, ke, ve, w, pos, bits, Hkv, D, n, page = args
    assert (bits == 8) == (ke is not None) == (k.dtype == torch.uint8) and k.shape == v.shape == (n, page, Hkv, D)
    assert all(x is None or x.shape == (n, page // 16, Hkv) for x in (ke, ve)) and all(x is None or x.shape == (Hkv, n * page) for x in (w, pos))
    return [x for x in (k, v, ke, ve) if x is not None] + [x.view(Hkv, n, page).transpose(0, 1) for x in (w, pos) if x is not None]


def _copy(*args):
    pairs, n, status = args[11:]
    pairs = pairs.tolist()
    assert len(pairs) == n and len({b for _, b in pairs}) == n and not {a for a, _ in pairs} & {b for _, b in pairs}
    for x in _arrays(args[:11]):
        for a, b in pairs:
            x[b] = x[a].clone()
    status.fill_(0)


def _compact(*args):
    table, max_pages, held, B, refs, new_id, status, _ = args[11:]
    old = refs.tolist()
    for p, r in enumerate(old):  # what the table says is what is counted
        assert r == sum(table[b, :held[b]].tolist().count(p) for b in range(B))
    used = [p for p, r in enumerate(old) if r]
    gaps = [p for p in range(len(used)) if not old[p]]
    to = {p: p for p in used if p < len(used)}
    to.update(zip([p for p in used if p >= len(used)], gaps))
    for x in _arrays(args[:11]):
        for a, b in to.items():
            x[b] = x[a].clone()
    for b in range(B):
        for i in range(int(held[b])):
            table[b, i] = to[int(table[b, i])]
    new_id.copy_(torch.tensor([to.get(p, -1) for p in range(len(old))], dtype=torch.int32))
    status.fill_(0)


def _append(*args):
    k, _, v, _, dtype, off, B, T, Hkv, D, kc, vc, ke, ve, n, page, table, _, ctx, status = args
    assert k.dtype == {rs.RS_BF16: torch.bfloat16, rs.RS_F16: torch.float16}[dtype] and k.shape == (T, Hkv, D)
    for c, e, x in ((kc, ke, k), (vc, ve, v)):
        cr.append(c, e, table.tolist(), x, off.tolist(), ctx.tolist(), page)
    status.fill_(0)


@pytest.fixture(autouse=True)
def _calls(monkeypatch):
    monkeypatch.setattr(rs, "rs_pages_copy", _copy)
    monkeypatch.setattr(rs, "rs_pages_compact", _compact)
    monkeypatch.setattr(rs, "rs_pages_compact_workspace_size", lambda n: 4 * n)
    monkeypatch.setattr(rs, "rs_coded_append", _append)


def _cache(B=4, tokens=200, page=16, pages=40, **kw):
    return SharedCache(B, tokens, page, 2, 64, pages, device="cpu", **kw)


def _write(c, b, at, tags):
    """Tokens `tags` to request b's slots from at on, in every array that the cache has."""
    rows = c.rows(b, torch.arange(at, at + len(tags)))
    t = torch.tensor(tags)
    for x in (c.k, c.v):
        x.view(-1, 2, 64)[rows] = (t % 251).to(x.dtype)[:, None, None]
    if c.weights is not None:
        c.weights[:, rows] = t.float()
        c.positions[:, rows] = t.int()
    if c.bits == 8:
        c.k_exps.view(-1, 2)[rows // 16] = (t % 100).to(torch.int8)[:, None]


def _read(c, b, n):
    rows = c.rows(b, torch.arange(n))
    out = [c.k.view(-1, 2, 64)[rows][:, 1, 5].long(), c.v.view(-1, 2, 64)[rows][:, 0, 63].long()]
    if c.weights is not None:
        out += [c.weights[1, rows].long(), c.positions[0, rows].long()]
    return [x.tolist() for x in out]


@pytest.mark.parametrize("kw", [dict(), dict(bits=8), dict(track_weights=True), dict(dtype=torch.float16, page=64, pages=14)])
@pytest.mark.parametrize("seed", range(6))
def test_requests_keep_their_tokens_whatever_is_done_to_others(kw, seed):
    c, g, tag = _cache(**kw), random.Random(seed), 0
    tokens = [[] for _ in range(4)]
    done = set()
    for _ in range(150):
        what = g.choice(["add", "add", "add", "fork", "fork", "free", "trim", "compact", "resize"])
        b = g.randrange(4)
        counts = [g.choice([0, 1, 5, 16, 30]) if g.random() < 0.5 else 0 for _ in range(4)]
        try:
            if what == "add" and all(len(t) + n <= 200 for t, n in zip(tokens, counts)):
                c.reserve(counts)
                for x, n in enumerate(counts):
                    new = list(range(tag, tag + n))
                    tag += n
                    _write(c, x, len(tokens[x]), [y % 251 for y in new])
                    tokens[x] += [y % 251 for y in new]
                c.advance(counts)
            elif what == "fork":
                to = [x for x in range(4) if not c.held[x] and x != b]
                n = len(tokens[b]) if c.weights is not None or g.random() < 0.5 else g.randrange(len(tokens[b]) + 1)
                c.fork(b, to, n)
                for x in to:
                    tokens[x] = tokens[b][:n]
            elif what == "free":
                c.free(b)
                tokens[b] = []
            elif what == "trim":
                c.trim(b)
            elif what == "compact":
                used = c.compact()
                assert used == len({p for h in c.held for p in h}) and all(p < used for h in c.held for p in h)
            elif what == "resize":
                used = c.n_pages - c.free_pages
                c.resize(used + g.choice([0, 3, 20]))
            done.add(what)
        except MemoryError:
            done.add("full")
        assert c.lengths == [len(t) for t in tokens] == c.seen and c.length.tolist() == c.lengths
        names = [p for h in c.held for p in h]
        assert c.refs == [names.count(p) for p in range(c.n_pages)] and sorted(c._free) == [p for p in range(c.n_pages) if p not in names]
        for x in range(4):
            assert c.table[x].tolist() == c.held[x] + [-1] * (c.max_pages - len(c.held[x]))
            for got in _read(c, x, len(tokens[x])):
                assert got == tokens[x]
    assert done >= {"add", "fork", "free", "trim", "compact", "resize"}
    c.check()


def test_new_tokens_never_go_to_a_shared_page():
    c = _cache()
    c.reserve([40, 0, 0, 0])
    c.advance([40, 0, 0, 0])
    c.fork(0, [1, 2])
    c.fork(0, [3], 20)
    assert [len(set(c.held[0]) & set(c.held[b])) for b in (1, 2, 3)] == [2, 2, 1]
    c.reserve([3, 3, 40, 3])
    for b in range(4):
        own = {c.held[b][s // 16] for s in range(c.lengths[b], c.lengths[b] + 3)}
        assert all(c.refs[p] == 1 for p in own)
    assert c.lengths == [40, 40, 40, 20]
    tracked = _cache(track_weights=True)
    tracked.reserve([40, 0, 0, 0])
    tracked.advance([40, 0, 0, 0])
    tracked.fork(0, [3])
    assert not set(tracked.held[0]) & set(tracked.held[3])


def test_what_the_pool_cannot_hold_takes_nothing():
    c = _cache(pages=5)
    c.reserve([30, 10, 0, 0])
    c.advance([30, 10, 0, 0])
    for counts in ([0, 0, 20, 20], [1, 30, 1, 0]):
        with pytest.raises(MemoryError, match="2 of 5 free"):
            c.reserve(counts)
    assert c.free_pages == 2 and [len(h) for h in c.held] == [2, 1, 0, 0]
    c.fork(0, [2, 3])
    c.free(1)
    assert c.free_pages == 1
    c.reserve([3, 0, 0, 0])  # to 33 tokens
    with pytest.raises(MemoryError, match="0 of 5 free"):
        c.fork(0, [1])
    assert c.lengths == [30, 0, 30, 30] and not c.held[1]


def test_a_request_may_fill_its_last_page():
    c = _cache()  # 200 tokens: 13 pages of 16
    c.reserve([30, 0, 0, 0])
    c.advance([30, 0, 0, 0])
    c.reserve([171, 0, 0, 0])
    assert c.slots(0) == 208


@pytest.mark.parametrize("call,word", [
    (lambda c: c.fork(0, [1]), "dsts"), (lambda c: c.fork(0, [2, 2]), "dsts"), (lambda c: c.fork(0, [0]), "dsts"), (lambda c: c.fork(0, [4]), "request 4"),
    (lambda c: c.fork(-1, [2]), "request -1"), (lambda c: c.fork(0, [2], 31), "n=31"), (lambda c: c.fork(0, [2], -1), "n=-1"),
    (lambda c: c.reserve([1, 2]), "counts"), (lambda c: c.reserve([179, 0, 0, 0]), "counts"), (lambda c: c.reserve([0, -1, 0, 0]), "counts"),
    (lambda c: c.advance([19, 0, 0, 0]), "counts"), (lambda c: c.keep(0, [18]), "nodes"), (lambda c: c.keep(2, [0]), "nodes"),
    (lambda c: c.free(4), "request 4"), (lambda c: c.trim(-1), "request -1"), (lambda c: c.resize(2), "pages=2"), (lambda c: c.resize(1 << 28), "slots"),
])
def test_refusals_change_nothing(call, word):
    c = _cache()
    c.reserve([30, 10, 0, 0])
    c.advance([30, 10, 0, 0])
    before = [list(h) for h in c.held], list(c.refs), list(c._free), list(c.lengths), c.table.tolist()
    with pytest.raises(ValueError, match=word):
        call(c)
    assert before == ([list(h) for h in c.held], list(c.refs), list(c._free), list(c.lengths), c.table.tolist())


def test_a_part_of_a_tracked_request_is_not_forked():
    c = _cache(track_weights=True)
    c.reserve([30, 0, 0, 0])
    c.advance([30, 0, 0, 0])
    with pytest.raises(ValueError, match="n=20"):
        c.fork(0, [1], 20)


@pytest.mark.parametrize("bad,word", [
    (dict(bits=8, track_weights=True), "bits=8"), (dict(bits=4), "bits=4"), (dict(bits=8, page_size=8), "page_size=8"), (dict(pages=-1), "pages=-1"),
    (dict(pages=1 << 28), "slots"), (dict(dtype=torch.float32), "dtype"),
])
def test_caches_that_no_call_would_take(bad, word):
    args = dict(dict(B=2, tokens=40, page_size=16, Hkv=2, D=64, pages=6, device="meta"), **bad)
    with pytest.raises(ValueError, match=word):
        SharedCache(**args)
    if "pages" not in bad:
        args.pop("pages")
        with pytest.raises(ValueError, match=word):
            PagedCache(**args)


# ------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_the_accepted_path_is_appended_anew(dt):
    c = PagedCache(2, 64, 16, 2, 64, dtype=dt, device="cpu", bits=8)
    c.advance([20, 5])
    k, v = (torch.randn(12, 2, 64, generator=torch.Generator().manual_seed(s)).to(dt) for s in (1, 2))
    c.append(k, v, torch.tensor([0, 9, 12], dtype=torch.int32), torch.zeros(12, dtype=torch.int32))
    at = c.rows(0, torch.tensor([20, 23, 28]))
    k3, v3 = c.values(at)
    want = [x.clone() for x in c._arrays()]
    for codes, e, x in ((want[0], want[2], k3), (want[1], want[3], v3)):
        cr.append(codes, e, c.table.tolist(), x, [0, 3, 3], c.lengths, 16)
    c.keep(0, [0, 3, 8])
    assert all(torch.equal(a, b) for a, b in zip(c._arrays(), want))
    c.keep(1, [])
    c.keep(1, [1])
    assert torch.equal(c.values(c.rows(1, torch.tensor([5])))[0], c.values(c.rows(1, torch.tensor([6])))[0])
    now = c.values(c.rows(0, torch.arange(20, 23)))
    for a, b in zip(now, (k3, v3)):  # the block's exponent is what it was, or its values were alone in a finer one
        assert torch.equal(a, b)


def test_values_are_codes_times_powers_of_two():
    c = PagedCache(1, 32, 32, 2, 64, dtype=torch.float16, device="cpu", bits=8)
    g = torch.Generator().manual_seed(5)
    c.k.copy_(torch.randint(0, 256, c.k.shape, generator=g))
    c.v.copy_(c.k.flip(1) & 0xbf)
    c.k_exps.copy_(torch.randint(-15, 0, c.k_exps.shape, generator=g))
    c.v_exps.fill_(100)  # counts as 8
    k, v = c.values(c.rows(0, torch.arange(32)))
    assert torch.equal(k.double().nan_to_num(7e5), cr.values(c.k, c.k_exps)[0].nan_to_num(7e5))
    assert torch.equal(v.double(), cr.values(c.v, c.v_exps.clamp(max=8))[0])


def test_attention_says_how_many_rows_a_request_has(monkeypatch):
    got = []
    monkeypatch.setattr(rs, "rs_coded_attn_workspace_size", lambda B, T, most, *a: got.append((B, T, most)) or 100)

    def attn(q, stride, dtype, off, parents, B, T, most, Hq, Hkv, D, *rest):
        assert rest[2].dtype == torch.int8 and rest[-1].numel() >= 100
        got.append((B, T, most, Hq, Hkv, D))
        rest[-2].copy_(torch.tensor([0, rs.RS_ST_TOO_LARGE], dtype=torch.int32))

    monkeypatch.setattr(rs, "rs_coded_attn", attn)
    c = PagedCache(2, 64, 16, 2, 64, device="cpu", bits=8)
    q, off = torch.zeros(7, 4, 64, dtype=torch.bfloat16), torch.tensor([0, 2, 7], dtype=torch.int32)
    c.attend(q, off, 0.1)
    c.attend(q, off, 0.1, max_new=5)
    assert got == [(2, 7, 7), (2, 7, 7, 4, 2, 64), (2, 7, 5), (2, 7, 5, 4, 2, 64)]
    with pytest.raises(RuntimeError, match="request 1: TOO_LARGE"):
        c.check()
    for call in (lambda: c.weigh(q, torch.zeros(7, 4), off, 0.1), lambda: c.evict([9, 9], 4, 1)):
        with pytest.raises(ValueError, match="track_weights"):
            call()


def test_the_loop_in_8_bits_wants_pages_and_no_budget():
    from paper_2511_01282_gb300.e2e import SpecLoop
    for kw in (dict(), dict(cache="paged", budget=90)):
        with pytest.raises(ValueError, match="bits=8"):
            SpecLoop(None, None, [1], None, bits=8, **kw)


def test_a_trees_positions_are_its_depths():
    from paper_2511_01282_gb300.e2e import TinyLM
    m = TinyLM(V=16, d=64, L=1, Hq=1, Hkv=1, ffn=8, device="cpu", rotary=True)
    g = random.Random(2)
    for parents in ([-1], list(range(-1, 255)), [-1] + [g.randrange(i) for i in range(1, 256)]):
        depth = [0] * len(parents)
        for i, p in enumerate(parents):
            depth[i] = depth[p] + 1 if p >= 0 else 0
        assert m._positions(1000, torch.tensor(parents, dtype=torch.int32)).tolist() == [1000 + d for d in depth]


@pytest.mark.parametrize("kw", [dict(), dict(track_weights=True), dict(bits=8)])
@pytest.mark.parametrize("call", ["reserve", "fork", "trim", "free", "compact", "shrink", "grow", "advance"])
def test_a_call_that_fails_on_the_way_changes_nothing(kw, call, monkeypatch):
    """Whatever it makes of memory in turn, or the library's call, fails: lists, table, lengths and arrays stay as they were.  (A pool that
    could not be made smaller or larger may be closed up.)"""
    tokens = {0: list(range(37)), 1: list(range(100, 120))}

    def made():
        c = _cache(**kw)
        c.reserve([0, 30, 0, 0])
        c.reserve([50, 0, 0, 0])
        for b, t in tokens.items():
            _write(c, b, 0, t)
        c.advance([37, 20, 0, 0])
        return c

    def state(c):
        return (([list(h) for h in c.held], list(c.refs), list(c._free), list(c.lengths), list(c.seen), c.n_pages, c._size),
                [x.tolist() for x in (c.table, c.length, c.next)])

    def fails(name, at):
        """The at-th call of torch.<name> or of the library's call fails.  Whether it came to that."""
        c = made()
        before, left, owner = state(c), [at], rs if name.startswith("rs_") else torch
        whole = getattr(owner, name)

        def f(*a, **k):
            left[0] -= 1
            if left[0] == 0:
                raise RuntimeError("no memory")
            return whole(*a, **k)

        with monkeypatch.context() as m:
            m.setattr(owner, name, f)
            try:
                dict(reserve=lambda: c.reserve([40, 0, 30, 0]), fork=lambda: c.fork(0, [2, 3]), trim=lambda: c.trim(0), free=lambda: c.free(1),
                     compact=c.compact, shrink=lambda: c.resize(10), grow=lambda: c.resize(60), advance=lambda: c.advance([3, 1, 0, 0]))[call]()
            except RuntimeError:
                pass
            else:
                return False
        if call in ("shrink", "grow"):
            assert c.n_pages == c._size == 40 and all(x is None or x.shape[0] == 40 for x in c._arrays())
            assert all(x is None or x.shape[1] == 640 for x in (c.weights, c.positions))
        else:
            assert state(c) == before, (name, at)
        for b, t in tokens.items():
            rows = c.rows(b, torch.arange(len(t)))
            assert c.k.view(-1, 2, 64)[rows, 0, 0].long().tolist() == [x % 251 for x in t]
        assert c.table[0, :4].tolist() + c.table[1, :2].tolist() == c.held[0][:4] + c.held[1]
        assert all(c.refs[p] == 1 for p in c.held[0] + c.held[1]) and sorted(c._free + c.held[0] + c.held[1]) == list(range(40))
        return True

    assert sum(fails(name, at) for name in ("tensor", "zeros", "empty", "rs_pages_copy", "rs_pages_compact") for at in range(1, 8))
