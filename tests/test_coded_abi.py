"""Host checks of the 8-bit cache's, rotary's and the pages' calls, without a GPU: every refusal comes before a launch."""
import pytest

from paper_2511_01282_gb300 import build

P, BIG = 0x10000, 1 << 40  # an address that no call below comes to use
APPEND = dict(k=P, k_stride=256, v=P, v_stride=256, dtype=0, off=P, B=1, T=8, Hkv=2, D=128, kp=P, vp=P, ke=P, ve=P, n_pages=4, page=16,
              table=P, most=4, ctx=P, status=P, stream=None)
ATTN = dict(q=P, q_stride=512, dtype=0, off=P, parents=None, B=1, T=8, max_new=8, Hq=4, Hkv=2, D=128, kp=P, vp=P, ke=P, ve=P, n_pages=4,
            page=16, table=P, most=4, ctx=P, scale=0.1, out=P, lse=P, status=P, ws=P, wb=BIG, stream=None)
LONG = dict(ATTN, T=100, max_new=100)
ROTARY = dict(q=P, q_stride=512, qo=P, qo_stride=512, k=P, k_stride=256, ko=2 * P, ko_stride=264, dtype=1, pos=P, T=8, Hq=4, Hkv=2, D=128,
              rot=64, layout=0, turns=P, scale=1.0, inverse=0, stream=None)
POOL = dict(kp=P, vp=P, ke=None, ve=None, weights=None, positions=None, bits=16, Hkv=2, D=128, n_pages=4, page=16)
COPY = dict(POOL, pairs=P, n=3, status=P, stream=None)
COMPACT = dict(POOL, table=P, most=4, held=P, B=2, refs=P, new_id=P, status=P, ws=P, wb=BIG, stream=None)
INVALID, UNSUPPORTED, CAPACITY = 1, 2, 3


@pytest.fixture(scope="module")
def rs():
    build.build()
    from paper_2511_01282_gb300 import respec
    respec.lib()
    return respec


def call(rs, name, base, **kw):
    assert set(kw) <= set(base)
    n = rs.rs_launch_count()
    st = getattr(rs.lib(), name)(*dict(base, **kw).values())
    assert rs.rs_launch_count() == n
    return st, rs.rs_last_error()


SHARED = [
    (dict(page=24), UNSUPPORTED, "24"), (dict(page=8), UNSUPPORTED, "page size 8"), (dict(page=131072), UNSUPPORTED, "131072"),
    (dict(n_pages=-1), INVALID, "negative"), (dict(most=-1), INVALID, "negative"), (dict(n_pages=1 << 27), INVALID, "2^31"),
    (dict(most=1 << 27), INVALID, "2^31"), (dict(table=None), INVALID, "null request"), (dict(off=None), INVALID, "null request"),
    (dict(ctx=None), INVALID, "null request"), (dict(status=None), INVALID, "null request"), (dict(kp=None), INVALID, "null page"),
    (dict(ve=None), INVALID, "null page"), (dict(vp=P + 8), INVALID, "aligned"), (dict(D=96), UNSUPPORTED, "96"),
    (dict(dtype=2), INVALID, "dtype 2"), (dict(B=-1), INVALID, "negative"), (dict(T=-1), INVALID, "negative"),
    (dict(T=(1 << 30) + 1), INVALID, "2^30"), (dict(B=(1 << 28) + 1), INVALID, "B="),
]


@pytest.mark.parametrize("name,base", [("rs_coded_append", APPEND), ("rs_coded_attn", ATTN), ("rs_coded_attn", LONG)])
@pytest.mark.parametrize("bad,status,word", SHARED)
def test_cache_refusals(rs, name, base, bad, status, word):
    st, msg = call(rs, name, base, **bad)
    assert st == status and word in msg and name in msg


@pytest.mark.parametrize("name,base,bad,status,word", [
    ("rs_coded_append", APPEND, dict(k=None), INVALID, "null row"), ("rs_coded_append", APPEND, dict(v=P + 2), INVALID, "aligned"),
    ("rs_coded_append", APPEND, dict(k_stride=248), INVALID, "rows of k and v"), ("rs_coded_append", APPEND, dict(v_stride=260), INVALID, "multiple"),
    ("rs_coded_append", APPEND, dict(Hkv=0), INVALID, "Hkv=0"), ("rs_coded_append", APPEND, dict(Hkv=65536), INVALID, "Hkv=65536"),
    ("rs_coded_attn", ATTN, dict(max_new=-1), INVALID, "max_new=-1"), ("rs_coded_attn", ATTN, dict(Hq=5), UNSUPPORTED, "Hq=5"),
    ("rs_coded_attn", ATTN, dict(Hq=258), UNSUPPORTED, "128"), ("rs_coded_attn", ATTN, dict(scale=0.0), INVALID, "scale"),
    ("rs_coded_attn", ATTN, dict(scale=float("nan")), INVALID, "scale"), ("rs_coded_attn", ATTN, dict(out=P + 16), INVALID, "32-byte"),
    ("rs_coded_attn", ATTN, dict(ws=P + 16), INVALID, "32-byte"), ("rs_coded_attn", ATTN, dict(q_stride=504), INVALID, "q rows"),
    ("rs_coded_attn", ATTN, dict(q=P + 8), INVALID, "aligned"), ("rs_coded_attn", ATTN, dict(wb=64), CAPACITY, "workspace 64"),
    ("rs_coded_attn", LONG, dict(wb=64), CAPACITY, "workspace 64"), ("rs_coded_attn", LONG, dict(ws=None), CAPACITY, "workspace"),
    ("rs_coded_attn", ATTN, dict(B=4097), INVALID, "4096"), ("rs_coded_attn", ATTN, dict(B=4096, Hq=512, Hkv=512), UNSUPPORTED, "2^20"),
    ("rs_coded_attn", ATTN, dict(lse=None), INVALID, "null row"),
    ("rs_rotary", ROTARY, dict(T=-1), INVALID, "T=-1"), ("rs_rotary", ROTARY, dict(dtype=7), INVALID, "dtype 7"),
    ("rs_rotary", ROTARY, dict(D=100), UNSUPPORTED, "100"), ("rs_rotary", ROTARY, dict(D=520), UNSUPPORTED, "520"),
    ("rs_rotary", ROTARY, dict(rot=63), INVALID, "rot=63"), ("rs_rotary", ROTARY, dict(rot=130), INVALID, "rot=130"),
    ("rs_rotary", ROTARY, dict(rot=0), INVALID, "rot=0"), ("rs_rotary", ROTARY, dict(layout=2), INVALID, "layout 2"),
    ("rs_rotary", ROTARY, dict(scale=float("inf")), INVALID, "scale"), ("rs_rotary", ROTARY, dict(pos=None), INVALID, "null"),
    ("rs_rotary", ROTARY, dict(turns=None), INVALID, "null"), ("rs_rotary", ROTARY, dict(k=None), INVALID, "null row pointer (k)"),
    ("rs_rotary", ROTARY, dict(qo=None), INVALID, "null row pointer (q)"), ("rs_rotary", ROTARY, dict(q=P + 4), INVALID, "aligned"),
    ("rs_rotary", ROTARY, dict(k_stride=255), INVALID, "k rows of 255"), ("rs_rotary", ROTARY, dict(ko_stride=248), INVALID, "k_out rows"),
    ("rs_rotary", ROTARY, dict(qo_stride=1024), INVALID, "in place"), ("rs_rotary", ROTARY, dict(Hq=-1), INVALID, "Hq=-1"),
])
def test_other_refusals(rs, name, base, bad, status, word):
    st, msg = call(rs, name, base, **bad)
    assert st == status and word in msg and name in msg


@pytest.mark.parametrize("name,base", [("rs_pages_copy", COPY), ("rs_pages_compact", COMPACT)])
@pytest.mark.parametrize("bad,status,word", [
    (dict(bits=4), INVALID, "bits=4"), (dict(D=32), UNSUPPORTED, "32"), (dict(Hkv=0), INVALID, "Hkv=0"), (dict(page=12), UNSUPPORTED, "12"),
    (dict(bits=8, page=8), UNSUPPORTED, "page size 8"), (dict(n_pages=-1), INVALID, "negative"), (dict(kp=None), INVALID, "null page"),
    (dict(vp=P + 4), INVALID, "aligned"), (dict(bits=8), INVALID, "without exponents"), (dict(ke=P, ve=P), INVALID, "of a 16-bit"),
    (dict(Hkv=65535, page=65536), INVALID, "2^30"), (dict(status=None), INVALID, "null"),
])
def test_page_refusals(rs, name, base, bad, status, word):
    st, msg = call(rs, name, base, **bad)
    assert st == status and word in msg and name in msg


def test_the_rest(rs):
    for name, base, bad, status, word in [
        ("rs_pages_copy", COPY, dict(n=-1), INVALID, "n=-1"), ("rs_pages_copy", COPY, dict(pairs=None), INVALID, "null"),
        ("rs_pages_copy", COPY, dict(pairs=P + 4), INVALID, "8-byte"), ("rs_pages_compact", COMPACT, dict(B=-1), INVALID, "B=-1"),
        ("rs_pages_compact", COMPACT, dict(refs=None), INVALID, "null page"), ("rs_pages_compact", COMPACT, dict(held=None), INVALID, "null request"),
        ("rs_pages_compact", COMPACT, dict(table=None), INVALID, "null request"), ("rs_pages_compact", COMPACT, dict(most=-1), INVALID, "negative"),
        ("rs_pages_compact", COMPACT, dict(wb=16), CAPACITY, "workspace 16"), ("rs_pages_compact", COMPACT, dict(ws=P + 8), INVALID, "16-byte"),
    ]:
        st, msg = call(rs, name, base, **bad)
        assert st == status and word in msg and name in msg, (name, bad, st, msg)
    assert call(rs, "rs_coded_append", APPEND, B=0)[0] == 0 and call(rs, "rs_coded_attn", ATTN, B=0)[0] == 0
    assert call(rs, "rs_rotary", ROTARY, T=0)[0] == 0 and call(rs, "rs_rotary", ROTARY, Hq=0, Hkv=0)[0] == 0


def test_workspace_sizes(rs):
    f = rs.rs_coded_attn_workspace_size
    assert f(2, 2, 1, 8, 2, 128) > 0 and f(2, 100, 100, 8, 2, 128) == rs.rs_paged_attn_workspace_size(2, 100, 8, 2, 128)
    for bad in ((-1, 8, 1, 4, 4, 64), (1, -1, 1, 4, 4, 64), (1, 8, -1, 4, 4, 64), (1, 8, 1, 5, 2, 64), (1, 8, 1, 4, 4, 80), (4097, 8, 1, 4, 4, 64),
                (1, 8, 1, 256, 1, 64)):
        assert f(*bad) == 0
    assert rs.rs_pages_compact_workspace_size(1000) >= 4000 and rs.rs_pages_compact_workspace_size(-1) == 0
