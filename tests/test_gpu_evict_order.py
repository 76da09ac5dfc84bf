"""The order that rs_paged_evict keeps tokens in, where more are recent than the budget holds."""
import pytest
import torch

from test_gpu_evict import evict
from test_gpu_prompt_paged import _i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def test_recent_tokens_go_by_slot_and_the_others_by_weight():
    page, D = 8, 64
    kp, vp = (torch.zeros(2, page, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = _i32([[1, 0]])
    at = torch.tensor([8, 9, 10, 11, 12, 13, 14, 15, 0, 1], device="cuda")  # slots 0 to 9
    weight = torch.tensor([9.0, 1.0, float("inf"), 5.0, 7.0, 0.0, 8.0, 2.0, 3.0, 6.0], device="cuda")
    for position, budget, recent, kept in [
        ([0, 20, 2, 21, 22, 5, 23, 7, 24, 9], 3, 3, [1, 3, 4]),        # five recent: slots 1, 3, 4, 6, 8, whatever their weight
        ([0, 20, 2, 21, 22, 5, 23, 7, 24, 9], 6, 6, [1, 3, 4, 6, 8, 2]),  # ... and the heaviest of the others
        ([0, 1, 2, 3, 4, 5, 6, 7, 8, 9], 4, 0, [2, 0, 6, 4]),
    ]:
        w, pos = torch.zeros(1, 16, device="cuda"), torch.zeros(1, 16, dtype=torch.int32, device="cuda")
        w[0, at], pos[0, at] = weight, _i32(position)
        new, status = evict(kp, vp, page, table, [10], [20 + recent if recent else 10], budget, recent, w, pos)
        assert new == [budget] and status == [0]
        assert sorted(pos[0, at[:budget]].tolist()) == sorted(position[s] for s in kept)
