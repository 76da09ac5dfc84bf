"""A single token whose heads come from a [heads, 1, D] tensor: the same bits as from its own copy."""
import pytest
import torch

from test_gpu_paged_status import _cache, _i32, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def test_heads_of_one_token():
    from paper_2511_01282_gb300.paged import prompt_attention
    x, off = _rows(50), _i32(0, 1)
    results = []
    for form in (lambda t: t.transpose(0, 1).clone(memory_format=torch.contiguous_format).transpose(0, 1), lambda t: t.clone()):
        c = _cache(B=1)
        c.append(x, x, _i32(0, 50))
        c.advance([50])
        q, k, v = (form(_rows(1, heads=h, seed=s)) for h, s in ((4, 1), (2, 2), (2, 3)))
        c.append(k, v, off)
        out, lse = c.attend(q, off, 0.125)
        c.weigh(q, lse, off, 0.125)
        alone = prompt_attention(q, k, v, off, 0.125)
        c.check()
        results.append([out, lse, c.k, c.v, c.weights, alone[0], alone[1]])
    for a, b in zip(*results):
        assert torch.equal(a, b)
