"""Positions of tokens that a PagedCache numbers itself: behind an eviction, in a captured call, on the accepted path of a tree."""
import pytest
import torch

from test_gpu_paged_status import _cache, _i32, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _positions(c, b, first, n):
    return c.positions[:, c.rows(b, torch.arange(first, first + n, device="cuda"))].tolist()


def test_tokens_behind_an_eviction_are_recent():
    """Appended without positions they go on where the request is, not where its cache ends, and the next eviction keeps them."""
    c = _cache()
    x = _rows(240)
    c.append(x, x, _i32(0, 200, 240))
    c.advance([200, 40])
    c.weights.fill_(1.0)
    c.evict([200, 40], 64, 8)
    assert c.lengths == [64, 40]
    y = _rows(23)
    c.append(y, y, _i32(0, 20, 23))
    assert _positions(c, 0, 64, 20) == [list(range(200, 220))] * 2 and _positions(c, 1, 40, 3) == [[40, 41, 42]] * 2
    c.advance([20, 3])
    c.evict([220, 43], 64, 20)
    assert c.lengths == [64, 43]
    for p in _positions(c, 0, 0, 64):
        assert set(range(200, 220)) <= set(p)


def test_a_captured_append_goes_on_too():
    """The graph is taken before any eviction and replayed behind one."""
    c = _cache(B=1)
    x, one = _rows(100), _rows(3, seed=1)
    off, step = _i32(0, 100), _i32(0, 3)
    c.append(x, x, off)
    c.advance([100])
    c.append(one, one, step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.append(one, one, step)
    graph.replay()
    assert _positions(c, 0, 100, 3) == [[100, 101, 102]] * 2
    c.advance([3])
    c.weights.fill_(1.0)
    c.evict([103], 50, 10)
    graph.replay()
    assert _positions(c, 0, 50, 3) == [[103, 104, 105]] * 2


def test_the_accepted_path_of_a_tree_has_the_positions_that_follow():
    c = _cache()
    x = _rows(30)
    c.append(x, x, _i32(0, 20, 30))
    c.advance([20, 10])
    nodes = _rows(16, seed=1)
    c.append(nodes, nodes, _i32(0, 9, 16))
    c.keep(0, [0, 3, 8])
    c.keep(1, [0, 6])
    assert _positions(c, 0, 20, 3) == [[20, 21, 22]] * 2 and _positions(c, 1, 10, 2) == [[10, 11]] * 2
    # positions of the caller's own stay what they are
    c.append(nodes, nodes, _i32(0, 9, 16), _i32(*range(500, 516)))
    c.keep(0, [0, 3, 8])
    assert _positions(c, 0, 20, 3) == [[500, 503, 508]] * 2
