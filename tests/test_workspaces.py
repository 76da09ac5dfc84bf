"""Workspaces of the attention calls, without a GPU."""
import pytest

from paper_2511_01282_gb300 import build


@pytest.fixture(scope="module")
def rs():
    build.build()
    from paper_2511_01282_gb300 import respec
    return respec


@pytest.mark.parametrize("T", [1 << 10, 1 << 16])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_have_no_room_for_trees(rs, T, D):
    # 256 bits of ancestors a row are for the draft trees of rs_paged_attn
    prompt, paged = rs.rs_prompt_attn_workspace_size(3, T, 8, 2, D), rs.rs_paged_attn_workspace_size(3, T, 8, 2, D)
    assert paged - prompt >= 32 * T > 0
