"""PagedCache and the loop's cache handling on the host, without a GPU: the library's calls are stood in for where a test needs
their outputs."""
import pytest
import torch

from paper_2511_01282_gb300 import respec as rs
from paper_2511_01282_gb300.paged import PagedCache


def test_keep_refuses_tokens_that_no_page_holds():
    """Their table entries do not exist: on the device the lookup would be an index out of range."""
    c = PagedCache(2, 64, 16, 2, 64, device="cpu")
    c.advance([60, 3])
    before = c.k.clone()
    for b, nodes in ((0, [0, 4]), (0, [-1]), (0, [1 << 40]), (0, torch.tensor([0, 1, 9])), (1, [61]), (2, [0]), (-1, [0])):
        with pytest.raises(ValueError, match="request" if b in (2, -1) else "nodes"):
            c.keep(b, nodes)
    assert torch.equal(c.k, before)


def test_keep_takes_the_last_slot():
    c = PagedCache(2, 64, 16, 2, 64, device="cpu")
    c.k.view(-1, 2, 64)[:] = torch.arange(128, dtype=torch.bfloat16)[:, None, None]
    c.advance([60, 3])
    c.keep(0, [0, 3])
    c.keep(1, torch.tensor([2, 60]))
    c.keep(1, [])
    assert c.k.view(-1, 2, 64)[60:64, 0, 0].tolist() == [60, 63, 62, 63]
    assert c.k.view(-1, 2, 64)[64 + 3:64 + 6, 0, 0].tolist() == [64 + 5, 64 + 63, 64 + 5]


def _stub(monkeypatch, name, status, also=None):
    """rs.<name> leaves `status` in the tensor that follows what the call of the library has for it."""
    def call(*args):
        if also:
            also(*args)
        at = -1 if name == "rs_paged_append" else -2
        args[at].copy_(torch.tensor(status, dtype=torch.int32))
    monkeypatch.setattr(rs, name, call)
    if hasattr(rs, name + "_workspace_size"):
        monkeypatch.setattr(rs, name + "_workspace_size", lambda *a: 0)


def _tracked(B=2, **kw):
    return PagedCache(B, 64, 16, 2, 64, track_weights=True, device="cpu", **kw)


def _x(n, h=2):
    return torch.zeros(n, h, 64, dtype=torch.bfloat16)


OFF = torch.tensor([0, 2, 5], dtype=torch.int32)


def test_statuses_gather_until_they_are_looked_at(monkeypatch):
    c, q, lse = _tracked(), _x(5, 4), torch.zeros(5, 4)
    _stub(monkeypatch, "rs_paged_append", [0, rs.RS_ST_BAD_PAGE])
    c.append(_x(5), _x(5), OFF)
    _stub(monkeypatch, "rs_paged_append", [0, 0])
    c.append(_x(5), _x(5), OFF)
    _stub(monkeypatch, "rs_paged_attn", [0, rs.RS_ST_TIMEOUT])
    c.attend(q, OFF, 0.1)
    _stub(monkeypatch, "rs_paged_weights", [0, 0])
    c.weigh(q, lse, OFF, 0.1)
    with pytest.raises(RuntimeError, match="request 1: BAD_PAGE TIMEOUT$"):
        c.check()
    c.check()
    c.report(torch.tensor([1024, 0], dtype=torch.int32))
    with pytest.raises(RuntimeError, match="request 0: status 1024$"):
        c.check()


def test_an_eviction_takes_the_lengths_that_are_reported(monkeypatch):
    c = _tracked()
    c.advance([40, 30])

    def lengths(*args):
        args[-3].copy_(torch.tensor([40, 8], dtype=torch.int32))

    _stub(monkeypatch, "rs_paged_evict", [rs.RS_ST_BAD_PAGE, 0], lengths)
    with pytest.raises(RuntimeError, match="request 0: BAD_PAGE$"):
        c.evict([40, 30], 8, 2)
    assert c.lengths == [40, 8] and c.length.tolist() == [40, 8]


def test_tokens_without_positions_go_on_from_those_seen(monkeypatch):
    c, got = _tracked(B=3), []

    def evicted(*args):
        args[-3].copy_(torch.tensor([8, 8, 3], dtype=torch.int32))

    _stub(monkeypatch, "rs_paged_append", [0] * 3, lambda *a: got.append(a[4] if a[4] is None else a[4].tolist()))
    _stub(monkeypatch, "rs_paged_evict", [0] * 3, evicted)
    off = torch.tensor([0, 2, 2, 5], dtype=torch.int32)
    c.append(_x(7), _x(7), off)  # two rows behind the last request
    c.advance([40, 30, 3])
    c.evict([40, 30, 3], 8, 2)
    c.append(_x(5), _x(5), off)
    c.advance([2, 0, 1])
    c.append(_x(5), _x(5), off)
    own = torch.arange(5, dtype=torch.int32)
    c.append(_x(5), _x(5), off, own)
    c.append(_x(0), _x(0), torch.zeros(4, dtype=torch.int32))
    assert [x[:5] if x else x for x in got] == [[0, 1, 0, 1, 2], [40, 41, 3, 4, 5], [42, 43, 4, 5, 6], [0, 1, 2, 3, 4], None]
    assert c.lengths == [10, 8, 4] and c.seen == [42, 30, 4]
    assert c.length.tolist() == c.lengths and c.next.tolist() == c.seen
    plain = PagedCache(3, 64, 16, 2, 64, device="cpu")  # no positions to keep: nothing is computed for them
    plain.append(_x(5), _x(5), off)
    assert got[-1] is None


def test_offsets_that_decrease_number_nothing_out_of_range(monkeypatch):
    c = _tracked()
    _stub(monkeypatch, "rs_paged_append", [rs.RS_ST_BAD_OFFSET] * 2)
    for off in ([0, 9, 4], [-3, 2, 5], [7, 7, 7], [5, 0, -9]):
        c.append(_x(5), _x(5), torch.tensor(off, dtype=torch.int32))


def test_the_accepted_path_follows_on(monkeypatch):
    c = _tracked(B=1)
    _stub(monkeypatch, "rs_paged_append", [0])
    c.advance([20])
    off = torch.tensor([0, 9], dtype=torch.int32)
    c.append(_x(9), _x(9), off)
    c.positions[:, 20:29] = torch.arange(20, 29, dtype=torch.int32)
    c.keep(0, [0, 3, 8])
    assert c.positions[0, 20:24].tolist() == [20, 21, 22, 23]
    c.append(_x(9), _x(9), off, off.new_tensor(range(500, 509)))
    c.positions[:, 20:29] = torch.arange(500, 509, dtype=torch.int32)
    c.keep(0, [0, 3, 8])
    assert c.positions[0, 20:24].tolist() == [500, 503, 508, 503]


def test_a_refused_eviction_changes_nothing(monkeypatch):
    c = _tracked()
    c.advance([40, 30])

    def refused(*args):
        raise rs.RespecError(rs.RS_ERR_INVALID_ARG, "budget=0")

    _stub(monkeypatch, "rs_paged_evict", [0, 0], refused)
    with pytest.raises(rs.RespecError):
        c.evict([90, 90], 0, 0)
    assert (c.lengths, c.seen, c.length.tolist(), c.next.tolist()) == ([40, 30], [40, 30], [40, 30], [40, 30])


def test_a_single_row_has_no_distance_to_the_next(monkeypatch):
    """What a tensor says of the stride of a dimension of one row is anything: a token's heads taken from [heads, 1, D] say D."""
    from paper_2511_01282_gb300 import paged
    got = []
    c = PagedCache(1, 64, 16, 2, 64, device="cpu", track_weights=True)
    q, k = (torch.zeros(h, 1, 64, dtype=torch.bfloat16).transpose(0, 1) for h in (4, 2))
    assert q.stride(0) == 64 and q.is_contiguous()
    off = torch.tensor([0, 1], dtype=torch.int32)
    _stub(monkeypatch, "rs_paged_append", [0], lambda *a: got.append((a[1], a[3])))
    _stub(monkeypatch, "rs_paged_attn", [0], lambda *a: got.append(a[1]))
    _stub(monkeypatch, "rs_paged_weights", [0], lambda *a: got.append(a[1]))
    _stub(monkeypatch, "rs_prompt_attn", [0], lambda *a: got.append((a[1], a[3], a[5])))
    c.append(k, k, off, off[:1])
    out, lse = c.attend(q, off, 0.1)
    c.weigh(q, lse, off, 0.1)
    paged.prompt_attention(q, k, k, off, 0.1)
    assert got == [(128, 128), 256, 256, (256, 128, 128)]
    wide = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    c.append(wide[:, :2], wide[:, 2:4], torch.tensor([0, 3], dtype=torch.int32), torch.arange(3, dtype=torch.int32))
    assert got[-1] == (512, 512)


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=torch.float32), "dtype"), (dict(D=96), "96"), (dict(page_size=24), "page_size=24"), (dict(page_size=4), "page_size=4"),
    (dict(page_size=0), "page_size=0"), (dict(page_size=1 << 17), "page_size=131072"), (dict(Hkv=0), "Hkv=0"), (dict(B=-1), "B=-1"),
    (dict(tokens=-1), "tokens=-1"), (dict(tokens=1 << 31), "slots"),
])
def test_a_cache_that_no_call_would_take_is_refused(bad, word):
    args = dict(dict(B=2, tokens=40, page_size=16, Hkv=2, D=64, dtype=torch.bfloat16, device="meta"), **bad)
    with pytest.raises(ValueError, match=word):
        PagedCache(**args)
