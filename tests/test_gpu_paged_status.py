"""What the calls of a PagedCache report about requests is gathered and raised, also from captured calls."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(B=2, tokens=512, page=16, Hkv=2, D=64):
    from paper_2511_01282_gb300.paged import PagedCache
    return PagedCache(B, tokens, page, Hkv, D, track_weights=True)


def _rows(n, heads=2, D=64, seed=0):
    return torch.randn(n, heads, D, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def test_a_bad_page_is_not_lost_behind_later_calls():
    c = _cache()
    x, off = _rows(100), _i32(0, 60, 100)
    q = _rows(100, heads=4)
    c.append(x, x, off)
    c.check()
    good = int(c.table[0, 1])
    c.table[0, 1] = 1 << 20
    out, lse = c.attend(q, off, 0.125)
    c.table[0, 1] = good
    c.weigh(q, lse, off, 0.125)
    with pytest.raises(RuntimeError, match="request 0.*BAD_PAGE"):
        c.check()
    c.check()  # reported once
    graph = torch.cuda.CUDAGraph()
    c.table[1, 2] = -7
    with torch.cuda.graph(graph):
        c.attend(q, off, 0.125)
    c.check()
    graph.replay()
    c.table[1, 2] = c.n_pages - 1
    c.append(x, x, off)
    with pytest.raises(RuntimeError, match="request 1.*BAD_PAGE"):
        c.check()


def test_an_eviction_that_is_rejected_says_so():
    c = _cache()
    x = _rows(300)
    c.append(x, x, _i32(0, 200, 300))
    c.advance([200, 100])
    good = int(c.table[0, 3])
    c.table[0, 3] = -1
    with pytest.raises(RuntimeError, match="request 0.*BAD_PAGE"):
        c.evict([200, 100], 64, 8)
    assert c.lengths == [200, 64] and c.length.tolist() == [200, 64]  # the one that is left alone, and the other
    c.table[0, 3] = good
    c.evict([200, 100], 64, 8)
    assert c.lengths == [64, 64] and c.length.tolist() == [64, 64]
