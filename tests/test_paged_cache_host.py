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
