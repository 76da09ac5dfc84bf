"""Barriers of the attention core over the cache in 8 bits: each one that is initialised is also waited for and arrived at."""
import re

from test_source_barriers import WAITS, _arguments
from test_source_rules import _text


def test_no_barrier_without_a_waiter():
    s = _text("coded_core.cuh")
    barriers = set(re.findall(r"mbar_init\((?:&(\w+)\[|other)", s)) - {""}
    assert len(barriers) == 15 and "mbar_init(other," in s
    q_there = {"qready", "qfull"}  # the issuing warps' name for either
    for calls, names in ((WAITS, q_there), (r"\b(?:umma_commit|warp_arrive|mbar_arrive_cnt|mbar_expect_tx)\s*\(", set())):
        text = _arguments(s, calls)
        seen = set(re.findall(r"&(\w+)\[", text))
        if "q_there[" in text:
            seen |= names
        assert barriers <= seen, sorted(barriers - seen)
        assert re.search(r"\bother\b", text)


def test_every_barrier_has_its_place():
    """As many words in shared memory as barriers."""
    s = _text("coded_core.cuh")
    assert "kNumBars = 2 * kNR + 2 * kNC + 23" in s
    pairs = set(re.findall(r"mbar_init\(&(\w+)\[x\]", s))
    assert 2 * len(pairs) + 1 <= 23 and len(set(re.findall(r"mbar_init\(&(\w+)\[s\]", s))) == 4
