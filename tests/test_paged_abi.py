"""Host checks of the prompt and paged-cache calls, without a GPU: every refusal comes before a launch."""
import ctypes as C

import pytest
import torch

from paper_2511_01282_gb300 import build


@pytest.fixture(scope="module")
def rs():
    build.build()
    from paper_2511_01282_gb300 import respec
    respec.lib()
    return respec


P = 0x10000  # an address that no call below comes to use
BIG = 1 << 40
PROMPT = dict(q=P, q_stride=512, k=P, k_stride=256, v=P, v_stride=256, dtype=0, off=P, B=1, T=8, Hq=4, Hkv=2, D=128, scale=0.1, out=P,
              lse=P, status=P, ws=P, wb=BIG, stream=None)
APPEND = dict(k=P, k_stride=256, v=P, v_stride=256, pos=None, off=P, B=1, T=8, Hkv=2, D=128, kp=P, vp=P, n_pages=4, page=16, table=P,
              most=4, ctx=P, weights=None, positions=None, status=P, stream=None)
ATTN = dict(q=P, q_stride=512, dtype=0, off=P, parents=None, B=1, T=8, Hq=4, Hkv=2, D=128, kp=P, vp=P, n_pages=4, page=16, table=P, most=4,
            ctx=P, scale=0.1, out=P, lse=P, status=P, ws=P, wb=BIG, stream=None)
WEIGH = dict(q=P, q_stride=512, dtype=0, lse=P, off=P, B=1, T=8, Hq=4, Hkv=2, D=128, kp=P, n_pages=4, page=16, table=P, most=4, ctx=P,
             scale=0.1, weights=P, status=P, ws=P, wb=BIG, stream=None)
EVICT = dict(kp=P, vp=P, Hkv=2, D=128, n_pages=4, page=16, table=P, most=4, length=P, nxt=P, B=1, budget=8, recent=2, weights=P, positions=P,
             new=P, status=P, ws=P, wb=BIG, stream=None)
CALLS = dict(rs_prompt_attn=PROMPT, rs_paged_append=APPEND, rs_paged_attn=ATTN, rs_paged_weights=WEIGH, rs_paged_evict=EVICT)
INVALID, UNSUPPORTED, CAPACITY = 1, 2, 3


def call(rs, name, **kw):
    args = dict(CALLS[name])
    assert set(kw) <= set(args)
    args.update(kw)
    n = rs.rs_launch_count()
    st = getattr(rs.lib(), name)(*args.values())
    assert rs.rs_launch_count() == n
    return st, rs.rs_last_error()


ATTENTION = ("rs_prompt_attn", "rs_paged_attn", "rs_paged_weights")
PAGED = ("rs_paged_append", "rs_paged_attn", "rs_paged_weights", "rs_paged_evict")


@pytest.mark.parametrize("name", ATTENTION)
@pytest.mark.parametrize("bad,status,word", [
    (dict(D=96), UNSUPPORTED, "96"), (dict(Hq=5), UNSUPPORTED, "Hq=5"), (dict(Hkv=0), UNSUPPORTED, "Hkv=0"), (dict(Hq=0), UNSUPPORTED, "Hq=0"),
    (dict(Hq=129, Hkv=1), UNSUPPORTED, "128"), (dict(dtype=2), INVALID, "dtype 2"), (dict(dtype=-1), INVALID, "dtype -1"),
    (dict(B=-1), INVALID, "negative"), (dict(T=-1), INVALID, "negative"), (dict(B=4097), INVALID, "4096"),
    (dict(T=(1 << 30) + 1), INVALID, "2^30"),
    (dict(scale=0.0), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(off=None), INVALID, "null request"), (dict(status=None), INVALID, "null request"), (dict(q=None), INVALID, "null row"),
    (dict(lse=None), INVALID, "null row"), (dict(q=P + 8), INVALID, "aligned"), (dict(ws=P + 8), INVALID, "aligned"),
    (dict(q_stride=511), INVALID, "q rows of 511"), (dict(q_stride=516), INVALID, "multiple of 8"), (dict(q_stride=-512), INVALID, "q rows"),
    (dict(wb=64), CAPACITY, "workspace 64"), (dict(ws=None), CAPACITY, "workspace"),
])
def test_attention_refusals(rs, name, bad, status, word):
    st, msg = call(rs, name, **bad)
    assert st == status and word in msg and name in msg


@pytest.mark.parametrize("name", PAGED)
@pytest.mark.parametrize("bad,status,word", [
    (dict(page=24), UNSUPPORTED, "24"), (dict(page=4), UNSUPPORTED, "page size 4"), (dict(page=0), UNSUPPORTED, "page size 0"),
    (dict(page=131072), UNSUPPORTED, "131072"), (dict(n_pages=-1), INVALID, "negative"), (dict(most=-1), INVALID, "negative"),
    (dict(n_pages=1 << 27), INVALID, "2^31"), (dict(most=1 << 27), INVALID, "2^31"), (dict(table=None), INVALID, "null request"),
    (dict(kp=None), INVALID, "null page"), (dict(kp=P + 8), INVALID, "aligned"), (dict(D=32), UNSUPPORTED, "32"),
    (dict(status=None), INVALID, "null request"),
])
def test_page_refusals(rs, name, bad, status, word):
    st, msg = call(rs, name, **bad)
    assert st == status and word in msg and name in msg


def test_other_refusals(rs):
    for name, bad, status, word in [
        ("rs_prompt_attn", dict(k=None), INVALID, "null row"), ("rs_prompt_attn", dict(v_stride=248), INVALID, "v rows of 248"),
        ("rs_prompt_attn", dict(out=P + 16), INVALID, "32-byte"), ("rs_prompt_attn", dict(k=P + 2), INVALID, "k must be"),
        ("rs_paged_attn", dict(out=P + 16), INVALID, "32-byte"), ("rs_paged_attn", dict(vp=None), INVALID, "null page"),
        ("rs_paged_attn", dict(ctx=None), INVALID, "null request"), ("rs_paged_append", dict(k_stride=8), INVALID, "rows of k and v"),
        ("rs_paged_append", dict(v=None), INVALID, "null row"), ("rs_paged_append", dict(Hkv=0), INVALID, "Hkv=0"),
        ("rs_paged_append", dict(v=P + 4), INVALID, "aligned"), ("rs_paged_append", dict(T=(1 << 30) + 1), INVALID, "2^30"),
        ("rs_paged_append", dict(B=(1 << 30) + 1), INVALID, "2^30"), ("rs_paged_weights", dict(weights=None), INVALID, "null page"),
        ("rs_paged_evict", dict(budget=0), INVALID, "budget=0"), ("rs_paged_evict", dict(recent=9), INVALID, "recent=9"),
        ("rs_paged_evict", dict(recent=-1), INVALID, "recent=-1"), ("rs_paged_evict", dict(positions=None), INVALID, "null page"),
        ("rs_paged_evict", dict(B=4096, Hkv=16), INVALID, "65535"), ("rs_paged_evict", dict(nxt=None), INVALID, "null request"),
        ("rs_paged_evict", dict(wb=8), CAPACITY, "workspace"),
    ]:
        st, msg = call(rs, name, **bad)
        assert st == status and word in msg and name in msg, (name, bad, st, msg)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_no_requests_is_no_work(rs, name):
    # (everything else is still checked)
    kw = dict(B=0)
    assert call(rs, name, **kw)[0] == 0
    assert call(rs, name, B=0, D=12)[0] == UNSUPPORTED


def test_workspace_sizes(rs):
    for f in (rs.rs_prompt_attn_workspace_size, rs.rs_paged_attn_workspace_size, rs.rs_paged_weights_workspace_size):
        assert f(2, 100, 8, 2, 128) > 0 and f(0, 0, 8, 2, 64) > 0
        for bad in ((-1, 8, 4, 4, 64), (1, -1, 4, 4, 64), (1, 8, 5, 2, 64), (1, 8, 4, 4, 80), (4097, 8, 4, 4, 64), (1, 8, 0, 4, 64),
                    (1, 8, 256, 1, 64)):
            assert f(*bad) == 0
    assert rs.rs_paged_evict_workspace_size(4, 8, 100) >= 4 * 8 * 100 * 8
    for bad in ((-1, 8, 1), (1, 0, 1), (1, 8, 0), (4097, 1, 1), (4096, 16, 4)):
        assert rs.rs_paged_evict_workspace_size(*bad) == 0


def test_rows_of_the_binding(rs):
    args = list(PROMPT.values())
    args = args[:-2] + args[-1:]  # the workspace tensor stands for (pointer, bytes)
    args[-2], args[-1] = None, 0
    with pytest.raises(rs.RespecError, match="workspace"):
        rs.rs_prompt_attn(*args)
    with pytest.raises(ValueError, match="CUDA"):
        rs.rs_prompt_attn(torch.zeros(8, 4, 128, dtype=torch.bfloat16), *args[1:])
    with pytest.raises(C.ArgumentError):
        rs.rs_prompt_attn(*[1.5 if i == 1 else a for i, a in enumerate(args)])


def test_refusals_of_the_cache():
    """Tensors that do not fit the cache are refused before the library sees their addresses."""
    from paper_2511_01282_gb300.paged import PagedCache, prompt_attention
    c = PagedCache(2, 40, 16, 2, 64, device="cpu")
    x = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    off, off3 = x(3, dt=torch.int32), x(4, dt=torch.int32)
    q, k, lse = x(5, 4, 64), x(5, 2, 64), x(5, 4, dt=torch.float32)
    for f, word in [
        (lambda: c.append(x(5, 2, 64, dt=torch.float16), k, off), "k:"), (lambda: c.append(k, x(5, 4, 64), off), "v:"),
        (lambda: c.append(k, x(4, 2, 64), off), "v: 5 rows"), (lambda: c.append(x(5, 2, 128), k, off), "k:"),
        (lambda: c.append(k, k, off3), "new_off"), (lambda: c.append(k, k, off.long()), "new_off"),
        (lambda: c.append(k, k, off, x(4, dt=torch.int32)), "pos"), (lambda: c.attend(q.half(), off, 0.1), "q:"),
        (lambda: c.attend(x(5, 4, 128), off, 0.1), "q:"), (lambda: c.attend(q, off, 0.1, x(6, dt=torch.int32)), "parents"),
        (lambda: c.attend(q, off3, 0.1), "new_off"), (lambda: c.weigh(q, lse[:, :2], off, 0.1), "lse"),
        (lambda: c.weigh(q, lse, off, 0.1), "track_weights"), (lambda: c.evict([1, 1], 8, 0), "track_weights"),
        (lambda: c.evict([1], 8, 0), "next_pos"), (lambda: c.advance([1]), "counts"), (lambda: c.advance([0, -1]), "counts"),
        (lambda: c.advance([49, 0]), "counts"), (lambda: prompt_attention(q, k.half(), k, off, 0.1), "k:"),
        (lambda: prompt_attention(q, k, x(5, 4, 64), off, 0.1), "v:"), (lambda: prompt_attention(q, k[:4], k[:4], off, 0.1), "k: 5 rows"),
        (lambda: prompt_attention(q, k, k, off.long(), 0.1), "seq_off"), (lambda: prompt_attention(q.float(), k, k, off, 0.1), "q:"),
    ]:
        with pytest.raises(ValueError, match=word):
            f()
    c.advance([48, 0])
    assert c.lengths == [48, 0] and c.length.tolist() == [48, 0]


def test_refusals_of_the_loop():
    from paper_2511_01282_gb300.e2e import SpecLoop
    for budget, recent in ((32, 64), (8, -1)):
        with pytest.raises(ValueError, match="recent=%d" % recent):
            SpecLoop(None, None, None, None, cache="paged", budget=budget, recent=recent)
