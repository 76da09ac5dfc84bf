"""Barriers of the attention and weight kernels: each one that is initialised is also waited for and arrived at."""
import re

import pytest

from test_source_rules import _text

WAITS = r"\b(?:mbar_wait|warp_wait|quick_wait|quick_wait2|wait)\s*\("


def _arguments(s, calls):
    """The text between the brackets of every call that the pattern finds."""
    out = []
    for m in re.finditer(calls, s):
        depth, i = 1, m.end()
        while depth:
            depth += (s[i] == "(") - (s[i] == ")")
            i += 1
        out.append(s[m.end():i - 1])
    return " ; ".join(out)


@pytest.mark.parametrize("name", ["flash.cuh", "weigh.cu"])
def test_no_barrier_without_a_waiter(name):
    s = _text(name)
    barriers = set(re.findall(r"mbar_init\(&(\w+)\[", s))
    assert len(barriers) >= 10
    waited = _arguments(s, WAITS)
    arrived = _arguments(s, r"\b(?:umma_commit|warp_arrive|mbar_arrive_cnt|mbar_expect_tx)\s*\(")
    aliases = dict(full=("kfull", "vfull"), empty=("kempty", "vempty")) if name == "flash.cuh" else {}
    for used in (waited, arrived):
        seen = set(re.findall(r"&(\w+)\[", used))
        for a, of in aliases.items():  # the copy warps' names for theirs
            if a in seen:
                seen |= set(of)
        assert barriers <= seen, sorted(barriers - seen)
