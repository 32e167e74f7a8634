"""Sizes that the library refuses are refused by the binding too, before anything of such a size is allocated (no GPU)."""
import pytest

from paper_2410_01623_amd import fira, training


@pytest.mark.parametrize("rotated", [-2, 0, 1, 7, (1 << 16) + 2, 1 << 40, 1 << 62])
def test_rotary_frequencies(rotated):
    with pytest.raises(fira.FiraError) as refused:
        training.fira_rotary_frequencies(rotated, device="cpu")
    assert refused.value.status == fira.FIRA_ERR_SHAPE


def test_the_largest_and_smallest():
    for rotated in (2, 1 << 16):
        f, scale = training.fira_rotary_frequencies(rotated, device="cpu")
        assert f.shape == (rotated // 2,) and float(f[0]) == 1.0 and scale == 1.0
