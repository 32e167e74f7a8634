"""Lists of AdamW states with one of them missing are refused: a checkpoint would go on from zeros without a word (no GPU)."""
import pytest
import torch

from paper_2410_01623_amd import fira, training


def codes():
    return torch.zeros(300, dtype=torch.uint8).view(torch.float8_e4m3fn)


@pytest.mark.parametrize("given", [
    lambda: {"m": [codes()], "v": [codes()], "m_scale": [None], "v_scale": [None]}, lambda: {"m": [codes()], "v": [codes()], "m_scale": [torch.zeros(2)], "v_scale": [None]},
    lambda: {"m": [codes()], "v": [codes()], "m_scale": [None], "v_scale": [torch.zeros(2)]}, lambda: {"m": [torch.zeros(300)], "v": [None]}, lambda: {"m": [None], "v": [torch.zeros(300)]},
    lambda: {"m": [None], "v": [None]}])
def test_a_missing_state(given):
    w = torch.zeros(300)
    with pytest.raises(fira.FiraError, match="in part"):
        training.AdamWList([w], [w], **given())


@pytest.mark.gpu
def test_scales_of_fp32_states_may_be_none():
    """As a list's own m_scale and v_scale have them."""
    w, g = ([torch.zeros(300, device="cuda:0") for _ in range(2)] for _ in range(2))
    first = training.AdamWList(w, g, state=[torch.float32, torch.float8_e4m3fn])
    again = training.AdamWList(w, g, m=first.m, v=first.v, m_scale=first.m_scale, v_scale=first.v_scale, t=first.t)
    assert again.m_scale[0] is None and again.m_scale[1] is first.m_scale[1]
