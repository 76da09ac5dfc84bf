"""A paged KV cache in 8 bits, rotary positions, and pages that are copied and closed up: calls of a serving program.

A case is one call:

  append8  ``rs_coded_append``: keys and values of new tokens into e4m3 pages, an exponent of two for each 16 tokens and head
  attend8  ``rs_coded_attn``: a chunk of new tokens (a single one, a piece of a prompt, a draft tree) against those pages
  rotary   ``rs_rotary``: queries and keys turned by their positions, or turned back (the gradient)
  copy     ``rs_pages_copy``: pages copied by a list of pairs, with all that the cache keeps about them
  compact  ``rs_pages_compact``: a pool's used pages moved below its free ones, page tables and reference counts renumbered

Some channels of the keys are much larger than the others and some tokens' values much smaller, as in trained models; queries are
scaled per head so that some heads attend to a few keys and others to thousands.  Pages are handed out in random order, as an
allocator that has run for a while does.
"""
import math
import random

import torch

own = False

_DT = dict(bf16=torch.bfloat16, f16=torch.float16)
_E = dict(bf16=(-117, 120), f16=(-15, 8))  # the exponents that a cache of this type's values has
_BLOCK = 16


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # One decoding step of sixteen requests: their newest tokens enter the cache, most of them in the middle of a block.
        dict(name="append8-step", op="append8", B=16, n_lo=1, n_hi=1, ctx_lo=1021, ctx_hi=8190, Hkv=8, D=128, page=64, dtype="bf16"),
        # The prompts of eight requests enter the cache.
        dict(name="append8-prompts", op="append8", B=8, n_lo=500, n_hi=8000, ctx_lo=0, ctx_hi=0, Hkv=8, D=128, page=16, dtype="f16"),
        # A single token of one interactive request: latency.
        dict(name="attend8-one", op="attend8", B=1, n_lo=1, n_hi=1, ctx_lo=2048, ctx_hi=2048, Hq=32, Hkv=8, D=128, page=16, tree=False,
             dtype="bf16"),
        # Single tokens of a batch with ragged contexts.
        dict(name="attend8-step", op="attend8", B=64, n_lo=1, n_hi=1, ctx_lo=1024, ctx_hi=8191, Hq=32, Hkv=8, D=128, page=64, tree=False,
             dtype="bf16"),
        # Chunked prefill of long prompts: the next pieces, small pages, small heads.
        dict(name="attend8-chunk", op="attend8", B=4, n_lo=200, n_hi=1000, ctx_lo=4000, ctx_hi=32000, Hq=32, Hkv=8, D=64, page=16,
             tree=False, dtype="f16"),
        # Draft trees of four long requests, as many KV heads as query heads: the verify step, the largest cache.
        dict(name="attend8-tree", op="attend8", B=4, n_lo=65, n_hi=65, ctx_lo=32768, ctx_hi=32768, Hq=40, Hkv=40, D=128, page=128,
             tree=True, dtype="bf16"),
        # One decoding step's queries and keys.
        dict(name="rotary-step", op="rotary", T=64, Hq=32, Hkv=8, D=128, rot=128, pairs="half", far=32768, factor=1.0, inverse=False,
             dtype="bf16"),
        # The rows of a pass over prompts, half of each head, positions scaled for long contexts.
        dict(name="rotary-prompts", op="rotary", T=16384, Hq=32, Hkv=8, D=128, rot=64, pairs="interleaved", far=131072, factor=8.0,
             inverse=False, dtype="f16"),
        # The gradient of whole heads, an odd number of rows.
        dict(name="rotary-grad", op="rotary", T=4097, Hq=40, Hkv=40, D=64, rot=64, pairs="half", far=8192, factor=1.0, inverse=True,
             dtype="bf16"),
        # A decoding step forks sixteen sequences: the partly filled last page of each is copied.
        dict(name="copy-fork", op="copy", pages=2048, moved=16, Hkv=8, D=128, page=64, bits=8, weights=False, dtype="bf16"),
        # Whole prefixes are copied, with the weights and positions that eviction keeps.
        dict(name="copy-prefix", op="copy", pages=8192, moved=2500, Hkv=8, D=128, page=32, bits=16, weights=True, dtype="bf16"),
        # A pool of which long requests have left a third in use, closed up.
        dict(name="compact-pool", op="compact", pages=16384, used=0.35, B=48, Hkv=8, D=128, page=32, bits=16, weights=False, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append8", "append8", "attend8", "attend8", "attend8", "attend8", "rotary", "rotary", "copy", "compact"])
    while True:
        Hkv, G = rng.choice([1, 2, 4, 8, 16, 40]), rng.choice([1, 2, 3, 4, 7, 8])
        c = dict(op=op, Hkv=Hkv, D=rng.choice([64, 128]), dtype=rng.choice(["bf16", "f16"]))
        page = rng.choice([16, 32, 64, 128, 256])
        if op in ("append8", "attend8"):
            hi = _log_int(rng, 64, 32768) if rng.random() < 0.85 else 0
            n = rng.choice([1, 1, _log_int(rng, 1, 2048)]) if hi else _log_int(rng, 1, 4096)
            c.update(B=_log_int(rng, 1, 64), n_lo=max(1, n // rng.choice([1, 4])), n_hi=n, ctx_lo=hi // rng.choice([1, 8]), ctx_hi=hi,
                     page=page)
            if op == "attend8":
                c.update(Hq=Hkv * G, tree=n <= 200 and rng.random() < 0.4)
        elif op == "rotary":
            D = rng.choice([64, 80, 128, 256])
            c.update(T=_log_int(rng, 1, 16384), Hq=Hkv * G, D=D, rot=rng.choice([D, D, D // 2, D // 4, 20]),
                     pairs=rng.choice(["half", "interleaved"]), far=_log_int(rng, 512, 1 << 20), factor=rng.choice([1.0, 4.0, 8.0]),
                     inverse=rng.random() < 0.4)
        else:
            pages = _log_int(rng, 64, 20000)
            c.update(pages=pages, page=page, bits=rng.choice([8, 16]))
            c["weights"] = c["bits"] == 16 and rng.random() < 0.4
            c.update(dict(moved=_log_int(rng, 1, pages // 2)) if op == "copy" else dict(used=rng.uniform(0.05, 0.95), B=_log_int(rng, 1, 64)))
        w = work(c)
        pool = c.get("pages", 0) * page * Hkv * c["D"] * c.get("bits", 0) // 4
        rows = c.get("B", 1) * c.get("Hq", 0) * c.get("n_hi", 0) * (c.get("ctx_hi", 0) + c.get("n_hi", 0))  # of the padded plain form
        if c.get("Hq", 1) <= 64 and w["bytes"] <= 1.3e9 and w["flops"] <= 3.4e11 and pool <= 1 << 32 and rows <= 4e9:
            return c


# ------------------------------------------------------------------ sizes
def _spread(B, lo, hi):
    """B sizes from lo to hi, evenly spread, in a fixed mixed order (hi itself where there is one)."""
    at = sorted(range(B), key=lambda i: (i * 37) % 101)
    return [hi if B == 1 else lo + (hi - lo) * i // (B - 1) for i in at]


def _sizes(case):
    """(new tokens, tokens cached before them) of every request."""
    B = case["B"]
    return _spread(B, case["n_lo"], case["n_hi"]), _spread(B, case["ctx_lo"], case["ctx_hi"])[::-1]


def _page_bytes(case):
    """Bytes of one page, all arrays."""
    tokens = case["page"] * case["Hkv"]
    return tokens * case["D"] * case["bits"] // 4 + (tokens // 8 if case["bits"] == 8 else 0) + (8 * tokens if case["weights"] else 0)


def _used(case):
    return max(1, min(case["pages"] - 1, int(case["pages"] * case["used"])))


def work(case):
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    if op == "rotary":
        return dict(bytes=case["T"] * (4 * (case["Hq"] + Hkv) * D + 4), flops=3 * case["T"] * (case["Hq"] + Hkv) * case["rot"])
    if op == "copy":
        return dict(bytes=case["moved"] * (2 * _page_bytes(case) + 8), flops=0)
    if op == "compact":  # the used pages behind the first `used` ones, spread evenly
        moved = _used(case) * (1 - _used(case) / case["pages"])
        return dict(bytes=int(moved * 2 * _page_bytes(case) + 12 * case["pages"] + 8 * _used(case)), flops=0)
    n, ctx = _sizes(case)
    T = sum(n)
    if op == "append8":
        return dict(bytes=T * (6 * Hkv * D + Hkv // 8 + 4), flops=0)
    Hq = case["Hq"]
    pairs = sum(a * c + (a if case["tree"] else a * (a + 1) // 2) for a, c in zip(n, ctx))
    return dict(bytes=sum(a + c for a, c in zip(n, ctx)) * (2 * Hkv * D + Hkv // 8) + T * (4 * Hq * D + 4 * Hq), flops=4 * D * Hq * pairs)


# ------------------------------------------------------------------ inputs
def _trees(n, seed):
    """Parents of every request's nodes: a model tree, bushiest near the root, and chains of up to eight from the root."""
    g = random.Random(seed)
    out = []
    for N in n:
        model = (N + 1) // 2
        par = [-1] + [int(i * g.random() ** 2) for i in range(1, model)]
        for i in range(len(par), N):
            par.append(0 if (i - model) % 8 == 0 else i - 1)
        out += par[:N]
    return torch.tensor(out, dtype=torch.int32)


def _frequencies(rot, base, factor):
    """Radians a position; those of long waves divided by the factor, those of short ones kept, a ramp between."""
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        wave = 2 * math.pi / f
        keep = min(1.0, max(0.0, (8192.0 / wave - 1.0) / 3.0))
        out.append(f * (keep + (1 - keep) / factor))
    return torch.tensor(out, dtype=torch.float64)


def prepare(case, seed):
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    dt = _DT[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    cpu = random.Random(seed)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen, dtype=dt)  # noqa: E731
    bits = lambda *s: torch.randint(0, 256, s, device="cuda", generator=gen, dtype=torch.uint8)  # noqa: E731
    st = dict(case=case)
    if op == "rotary":
        T, heads = case["T"], case["Hq"] + Hkv
        qk = normal(T, heads, D)  # one projection's rows: queries, keys
        st.update(q=qk[:, :case["Hq"]], k=qk[:, case["Hq"]:], pos=torch.randint(0, case["far"], (T,), device="cuda", generator=gen).int(),
                  freq=_frequencies(case["rot"], 10000.0 if case["factor"] == 1.0 else 500000.0, case["factor"]).cuda(),
                  scale=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0,
                  q_out=torch.zeros(T, case["Hq"], D, dtype=dt, device="cuda"), k_out=torch.zeros(T, Hkv, D, dtype=dt, device="cuda"))
        return st
    P = case["page"]
    if op in ("copy", "compact"):
        pages = case["pages"]
        if case["bits"] == 8:
            st.update(kp=bits(pages, P, Hkv, D) & 0x7e, vp=bits(pages, P, Hkv, D) & 0xbf,
                      ke=bits(pages, P // _BLOCK, Hkv).view(torch.int8) >> 4, ve=bits(pages, P // _BLOCK, Hkv).view(torch.int8) >> 4)
        else:
            st.update(kp=normal(pages, P, Hkv, D), vp=normal(pages, P, Hkv, D), ke=None, ve=None)
        st.update(w=None, pos=None, status=i32([0]))
        if case["weights"]:
            st.update(w=torch.rand(Hkv, pages * P, device="cuda", generator=gen),
                      pos=torch.randint(0, 1 << 20, (Hkv, pages * P), device="cuda", generator=gen).int())
        order = list(range(pages))
        cpu.shuffle(order)
        if op == "copy":
            m = case["moved"]
            st["pairs"] = i32([[order[i], order[m + i]] for i in range(m)])
            return st
        # used pages anywhere in the pool, dealt out to the requests; one in eight belongs to two of them
        used = order[:_used(case)]
        B = min(case["B"], len(used))
        lists = [used[b::B] for b in range(B)]
        shared = used[::8]
        for i, page in enumerate(shared):
            lists[(i + 1) % B].append(page)
        most = max(len(x) for x in lists)
        refs = [0] * pages
        for x in lists:
            for page in x:
                refs[page] += 1
        st.update(B=B, most=most, table0=i32([x + [-1] * (most - len(x)) for x in lists]), held=i32([len(x) for x in lists]), refs0=i32(refs),
                  status=i32([0] * B))
        return st
    n, ctx = _sizes(case)
    B, T = case["B"], sum(n)
    off = [0]
    for a in n:
        off.append(off[-1] + a)
    need = [-(-(a + c) // P) for a, c in zip(n, ctx)]
    most, pages = max(need), sum(need) + 3
    order = list(range(pages))
    cpu.shuffle(order)
    table, at = [], 0
    for x in need:
        table += order[at:at + x] + [0] * (most - x)
        at += x
    st.update(off=i32(off), ctx=i32(ctx), T=T, n_max=max(n), keys_max=max(a + c for a, c in zip(n, ctx)), pages=pages, most=most,
              table=i32(table).view(B, most), status=i32([0] * B))
    loud = torch.exp(torch.randn(Hkv, D, device="cuda", generator=gen) * 0.8).to(dt)  # the keys' channels
    if op == "append8":
        quiet = torch.exp(torch.randn(T, 1, 1, device="cuda", generator=gen) * 0.7).to(dt)
        st.update(k=normal(T, Hkv, D) * loud, v=normal(T, Hkv, D) * quiet)
        st.update(kp=bits(pages, P, Hkv, D) & 0xfe, vp=bits(pages, P, Hkv, D) & 0xfe)  # no NaN
        st.update({x: torch.randint(-9, -5, (pages, P // _BLOCK, Hkv), device="cuda", generator=gen).to(torch.int8) for x in ("ke", "ve")})
        return st
    for name, e in (("k", "ke"), ("v", "ve")):  # a head's pages at a time, as they were appended
        codes = torch.empty(pages * P // _BLOCK, _BLOCK, Hkv, D, dtype=torch.uint8, device="cuda")
        exps = torch.empty(pages * P // _BLOCK, Hkv, dtype=torch.int8, device="cuda")
        for h in range(Hkv):
            x = normal(pages * P // _BLOCK, _BLOCK, D).float()
            x = x * loud[h].float() if name == "k" else x * torch.exp(torch.randn(x.shape[0], _BLOCK, 1, device="cuda", generator=gen) * 0.7)
            ex = _exponent(x.abs().amax((1, 2)), case["dtype"])
            codes[:, :, h] = _code(x, ex[:, None, None], case["dtype"])
            exps[:, h] = ex.to(torch.int8)
        st[name + "p"], st[e] = codes.view(pages, P, Hkv, D), exps.view(pages, P // _BLOCK, Hkv)
    Hq = case["Hq"]
    sharp = torch.exp(torch.rand(Hq, 1, device="cuda", generator=gen) * 1.8 - 0.7).to(dt)
    st.update(q=normal(T, Hq, D) * sharp, out=torch.zeros(T, Hq, D, dtype=dt, device="cuda"), lse=torch.zeros(T, Hq, device="cuda"),
              scale=D ** -0.5 / 1.4, parents=_trees(n, seed).cuda() if case["tree"] else None)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    from paper_2511_01282_gb300 import respec as rs
    c = st["case"]
    op, Hkv, D = c["op"], c["Hkv"], c["D"]
    dt = rs.RS_BF16 if c["dtype"] == "bf16" else rs.RS_F16
    if op == "rotary":
        from paper_2511_01282_gb300 import rotary
        if "turns" not in st:  # laid out once, beside the model's weights
            st["turns"] = rotary.turns(st["freq"])
        row = (c["Hq"] + Hkv) * D
        rs.rs_rotary(st["q"], row, st["q_out"], c["Hq"] * D, st["k"], row, st["k_out"], Hkv * D, dt, st["pos"], c["T"], c["Hq"], Hkv, D,
                     c["rot"], rs.RS_ROTARY_HALF if c["pairs"] == "half" else rs.RS_ROTARY_INTERLEAVED, st["turns"], st["scale"],
                     int(c["inverse"]))
        return dict(q=st["q_out"], k=st["k_out"])
    if op == "copy":
        rs.rs_pages_copy(st["kp"], st["vp"], st["ke"], st["ve"], st["w"], st["pos"], c["bits"], Hkv, D, c["pages"], c["page"], st["pairs"],
                         c["moved"], st["status"])
        return _pool(st, st["status"])
    if op == "compact":
        table, refs = st["table0"].clone(), st["refs0"].clone()
        if "ws" not in st:
            st["ws"] = torch.empty(rs.rs_pages_compact_workspace_size(c["pages"]), dtype=torch.uint8, device="cuda")
            st["new_id"] = torch.empty(c["pages"], dtype=torch.int32, device="cuda")
        rs.rs_pages_compact(st["kp"], st["vp"], st["ke"], st["ve"], st["w"], st["pos"], c["bits"], Hkv, D, c["pages"], c["page"], table,
                            st["most"], st["held"], st["B"], refs, st["new_id"], st["status"], st["ws"])
        return dict(_pool(st, st["status"]), table=table, refs=refs, new_id=st["new_id"])
    cache = (st["kp"], st["vp"], st["ke"], st["ve"], st["pages"], c["page"], st["table"], st["most"], st["ctx"])
    if op == "append8":
        rs.rs_coded_append(st["k"], Hkv * D, st["v"], Hkv * D, dt, st["off"], c["B"], st["T"], Hkv, D, *cache, st["status"])
        return _pool(st, st["status"])
    Hq = c["Hq"]
    if "ws" not in st:
        st["ws"] = torch.empty(rs.rs_coded_attn_workspace_size(c["B"], st["T"], st["n_max"], Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    rs.rs_coded_attn(st["q"], Hq * D, dt, st["off"], st["parents"], c["B"], st["T"], st["n_max"], Hq, Hkv, D, *cache, st["scale"], st["out"],
                      st["lse"], st["status"], st["ws"])
    return dict(out=st["out"], lse=st["lse"], status=st["status"])


def _pool(st, status):
    """The pool, 8-bit codes as the values they stand for (beside their exponents)."""
    f8 = lambda x: x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x  # noqa: E731
    return dict(k=f8(st["kp"]), v=f8(st["vp"]), k_exps=st["ke"], v_exps=st["ve"], weights=st.get("w"), positions=st.get("pos"), status=status)


# ------------------------------------------------------------------ the plain forms
def _two(e):
    """2^e in fp32, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponent(most, dtype):
    """The least exponent with most <= 448 2^e, in the type's range."""
    m, e = torch.frexp(most)  # most = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    return torch.where(most == 0, _E[dtype][0], e.int() - torch.where(m <= 0.875, 9, 8)).clamp(*_E[dtype])


def _code(x, e, dtype):
    x = x * _two(-e)
    if dtype == "f16":  # nothing that fp16 does not hold
        x = torch.where(e == _E["f16"][1], x.clamp(-240.0, 240.0), x)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _value(codes, exps):
    return codes.view(torch.float8_e4m3fn).float() * _two(exps)


def _rows(st, slots):
    """Rows of the pool that hold these slots [B, L] of the requests."""
    P = st["case"]["page"]
    page = st["table"].long().gather(1, (slots // P).clamp(max=st["most"] - 1))
    return page * P + slots % P


def _run_plain(st):
    c = st["case"]
    op, Hkv, D = c["op"], c["Hkv"], c["D"]
    if op == "rotary":
        angle = st["pos"].double()[:, None] * st["freq"]  # in 64 bits: far positions
        s = torch.sin(angle).float()[:, None] * (-st["scale"] if c["inverse"] else st["scale"])
        co = torch.cos(angle).float()[:, None] * st["scale"]
        half, rot = c["rot"] // 2, c["rot"]
        out = {}
        for name in ("q", "k"):
            x = st[name].float()
            y = x.clone()
            a, b = (slice(0, half), slice(half, rot)) if c["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
            y[..., a] = x[..., a] * co - x[..., b] * s
            y[..., b] = x[..., b] * co + x[..., a] * s
            out[name] = y.to(st[name].dtype)
        return out
    if op == "copy":
        src, dst = st["pairs"].long().unbind(1)
        _move(st, src, dst)
        return _pool(st, torch.zeros_like(st["status"]))
    if op == "compact":
        used = st["refs0"] > 0
        U, n = used.sum(), c["pages"]
        at = torch.arange(n, device="cuda")
        src, dst = at[used & (at >= U)], at[~used & (at < U)]
        new_id = torch.where(used, at, -1)
        new_id[src] = dst
        _move(st, src, dst)
        refs = st["refs0"].clone()
        refs[dst] = refs[src]
        refs[src] = 0
        live = torch.arange(st["most"], device="cuda") < st["held"][:, None]
        table = torch.where(live, new_id[st["table0"].long().clamp(min=0)].int(), st["table0"])
        return dict(_pool(st, torch.zeros_like(st["status"])), table=table, refs=refs, new_id=new_id.int())
    B, P, dtype = c["B"], c["page"], c["dtype"]
    off, ctx = st["off"].long(), st["ctx"].long()
    n = off[1:] - off[:-1]
    if op == "append8":
        row_of = torch.arange(st["T"], device="cuda")
        b = torch.searchsorted(off[1:].contiguous(), row_of, right=True)
        slot = ctx[b] + row_of - off[b]
        row = st["table"].long()[b, slot // P] * P + slot % P
        back = torch.arange(1, _BLOCK, device="cuda")  # cached tokens of the block that the request's first new token falls into
        old = ctx[:, None] - back
        live = (old >= 0) & (old // _BLOCK == (ctx // _BLOCK)[:, None]) & (n > 0)[:, None]
        old = _rows(st, old.clamp(min=0))[live]
        for x, pool, exps in ((st["k"], st["kp"], st["ke"]), (st["v"], st["vp"], st["ve"])):
            x, pool, exps = x.float(), pool.view(-1, Hkv, D), exps.view(-1, Hkv)
            most = torch.zeros(exps.shape, device="cuda").index_reduce_(0, row // _BLOCK, x.abs().amax(2), "amax")
            e = _exponent(most, dtype)
            before = exps.int()
            kept = torch.zeros(exps.shape[0], dtype=torch.bool, device="cuda")
            kept[old // _BLOCK] = True
            e = torch.where(kept[:, None], torch.maximum(e, before), e)
            o = old // _BLOCK
            pool[old] = (pool[old].view(torch.float8_e4m3fn).float() * _two(before[o] - e[o])[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            pool[row] = _code(x, e[row // _BLOCK][..., None], dtype)
            exps[row // _BLOCK] = e[row // _BLOCK].to(torch.int8)
        return _pool(st, torch.zeros_like(st["status"]))
    Hq, N, L = c["Hq"], st["n_max"], st["keys_max"]
    G = Hq // Hkv
    i, j = torch.arange(N, device="cuda"), torch.arange(L, device="cuda")
    rows = _rows(st, j.expand(B, L))
    kv = []
    for pool, exps in ((st["kp"], st["ke"]), (st["vp"], st["ve"])):
        x = _value(pool.view(-1, Hkv, D)[rows], exps.view(-1, Hkv)[rows // _BLOCK][..., None])
        kv.append(x.masked_fill_((j >= (ctx + n)[:, None])[..., None, None], 0.0).permute(0, 2, 1, 3))  # [B, Hkv, L, D]
    real = i < n[:, None]
    at = (off[:-1, None] + i).clamp(max=max(st["T"] - 1, 0))
    q = st["q"][at].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    see = j <= (ctx[:, None] + i)[..., None]
    if c["tree"]:
        par = st["parents"].long()[at]
        step = ((par[..., None] == i) | (i[:, None] == i)).float()  # [B, node, parent or itself]
        for _ in range(max(N - 1, 1).bit_length()):  # paths of twice the length
            step = (step @ step > 0).float()
        d = j - ctx[:, None, None]
        see = (d < 0) | ((d < N) & (step.gather(2, d.clamp(0, N - 1).expand(B, N, L)) > 0))
    see = see & (j < (ctx + n)[:, None])[:, None]
    s = torch.matmul(q, kv[0].transpose(2, 3)).mul_(st["scale"])
    s.view(B, Hkv, N, G, L).masked_fill_(~see[:, None, :, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = torch.exp_(s.sub_(m))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, kv[1]) / z
    lse = (m + torch.log(z)).view(B, Hkv, N, G).permute(0, 2, 1, 3).reshape(B, N, Hq)
    o = o.view(B, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)
    return dict(out=o[real].to(st["out"].dtype), lse=lse[real], status=torch.zeros_like(st["status"]))


def _move(st, src, dst):
    for name in ("kp", "vp", "ke", "ve"):
        if st[name] is not None:
            st[name][dst] = st[name][src]
    for name in ("w", "pos"):
        if st[name] is not None:
            x = st[name].view(st["case"]["Hkv"], st["case"]["pages"], -1)
            x[:, dst] = x[:, src]


# ------------------------------------------------------------------ the definition in 64 bits
def _decoded(codes):
    """What e4m3 codes stand for: sign, four bits of exponent (bias 7), three of fraction; no exponent: eighths of 2^-6."""
    x = codes.long()
    e, f = (x >> 3) & 15, (x & 7).double()
    value = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * torch.pow(2.0, (e - 7).double()))
    value = torch.where((x & 127) == 127, math.nan, value)
    return torch.where(x >= 128, -value, value)


def exact(case, seed):
    st = prepare(case, seed)
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    if op in ("copy", "compact"):  # copies and choices: nothing is computed that could be off
        return None
    if op == "rotary":
        out = {}
        sign = -1.0 if case["inverse"] else 1.0
        for name in ("q", "k"):
            y = st[name].double().clone()
            for i in range(case["rot"] // 2):
                a, b = (i, i + case["rot"] // 2) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
                turn = torch.polar(torch.full((case["T"],), st["scale"], dtype=torch.float64, device="cuda"),
                                   sign * st["pos"].double() * float(st["freq"][i]))
                z = torch.complex(st[name][..., a].double(), st[name][..., b].double()) * turn[:, None]
                y[..., a], y[..., b] = z.real, z.imag
            out[name] = y
        return out
    n, ctx, P = *_sizes(case), case["page"]
    off = [0]
    for a in n:
        off.append(off[-1] + a)

    def places(b, lo, hi):
        page = torch.tensor([int(p) for p in st["table"][b].cpu()], device="cuda").repeat_interleave(P) * P
        return (page + torch.arange(P, device="cuda").repeat(st["most"]))[lo:hi]

    if op == "append8":
        lo, hi = _E[case["dtype"]]
        out = {}
        for name in ("k", "v"):
            codes = _decoded(st[name + "p"].flatten(0, 1))
            exps = st[name + "e"].flatten(0, 1).long().clone()
            for b in range(case["B"]):
                x = st[name][off[b]:off[b + 1]].double()
                first = ctx[b] // _BLOCK * _BLOCK
                rows = places(b, first, ctx[b] + n[b])
                whole = torch.zeros(-(-rows.numel() // _BLOCK) * _BLOCK, Hkv, D, dtype=torch.float64, device="cuda")
                whole[ctx[b] - first:rows.numel()] = x
                top = whole.abs().view(-1, _BLOCK, Hkv, D).amax((1, 3))
                e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0) - 1e-12).long()
                e = torch.where(top > 448.0 * torch.pow(2.0, e.double()), e + 1, e).clamp(lo, hi)
                if ctx[b] > first:
                    e[0] = torch.maximum(e[0], exps[rows[0] // _BLOCK])
                    old = rows[:ctx[b] - first]
                    codes[old] = codes[old] * torch.pow(2.0, (exps[rows[0] // _BLOCK] - e[0]).double())[None, :, None]
                exps[rows[::_BLOCK] // _BLOCK] = e
                codes[rows[ctx[b] - first:]] = x * torch.pow(2.0, -e.double())[torch.arange(ctx[b] - first, rows.numel(), device="cuda") // _BLOCK][..., None]
            out[name] = codes.view(st[name + "p"].shape)
            out[name + "_exps"] = exps.view(st[name + "e"].shape)
        return dict(out, weights=None, positions=None, status=torch.zeros_like(st["status"]))
    if work(case)["flops"] > 4e12:  # about 20 seconds of fp64
        return None
    Hq, G = case["Hq"], case["Hq"] // Hkv
    out = torch.zeros(st["T"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["T"], Hq, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        rows = places(b, 0, ctx[b] + n[b])
        tree = None
        if case["tree"]:  # node j is seen by i where the walk up from i meets it
            tree = torch.zeros(n[b], n[b], dtype=torch.bool)
            par = st["parents"][off[b]:off[b + 1]].tolist()
            for i in range(n[b]):
                j = i
                while j >= 0:
                    tree[i, j] = True
                    j = par[j]
            tree = tree.cuda()
        for h in range(Hkv):
            k, v = (_decoded(st[x + "p"].flatten(0, 1)[rows, h]) *
                    torch.pow(2.0, st[x + "e"].flatten(0, 1)[rows // _BLOCK, h].double())[:, None] for x in ("k", "v"))
            for g in range(h * G, h * G + G):
                for i in range(0, n[b], 2048):
                    e = min(n[b], i + 2048)
                    last = ctx[b] + n[b] if tree is not None else ctx[b] + e  # no later key is seen
                    x = st["q"][off[b] + i:off[b] + e, g].double() @ k[:last].T * st["scale"]
                    hidden = torch.zeros(e - i, last, dtype=torch.bool, device="cuda")
                    if tree is not None:
                        hidden[:, ctx[b]:] = ~tree[i:e]
                    else:
                        hidden[:, ctx[b] + i:] = torch.ones(e - i, e - i, dtype=torch.bool, device="cuda").triu(1)
                    x[hidden] = -math.inf
                    z = torch.logsumexp(x, 1)
                    lse[off[b] + i:off[b] + e, g] = z
                    out[off[b] + i:off[b] + e, g] = torch.exp(x - z[:, None]) @ v[:last]
    return dict(out=out, lse=lse, status=torch.zeros_like(st["status"]))
