"""The decoding loop over paged caches stops at what its calls report."""
import pytest

from paper_2511_01282_gb300 import respec as rs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _loop(**kw):
    from paper_2511_01282_gb300.e2e import SpecLoop, TinyLM, make_prompt
    target = TinyLM(seed=0)
    draft = TinyLM(seed=1, base=target, noise=0.1)
    return SpecLoop(target, draft, make_prompt(target.V, 300, seed=2), rs.params(tau=0.0, span_len=8), cache="paged", **kw)


@pytest.mark.parametrize("which", ["tc", "dc"])
def test_the_loop_stops_at_a_bad_page(which):
    loop = _loop()
    loop.generate(4)
    getattr(loop, which)["layers"][1].table[0, 2] = 1 << 29
    with pytest.raises(RuntimeError, match="BAD_PAGE"):
        loop.generate(8)


def test_the_loop_stops_at_a_prompt_that_timed_out(monkeypatch):
    from paper_2511_01282_gb300 import e2e
    real = e2e.prompt_attention

    def late(*a):
        out, lse, status, ws = real(*a)
        return out, lse, status | rs.RS_ST_TIMEOUT, ws

    monkeypatch.setattr(e2e, "prompt_attention", late)
    with pytest.raises(RuntimeError, match="TIMEOUT"):
        _loop()
