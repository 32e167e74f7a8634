"""Clipping where the norm leaves the range of fp32: what the caller is told and what is done to the gradients agree."""
import math

import pytest
import torch

from paper_2410_01623_amd import training

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("limit", [0.0, 1.0, 3e38])
def test_a_norm_beyond_fp32_leaves_the_gradients(limit):
    """Finite values whose norm fp32 does not hold: the caller reads inf, and inf leaves the gradients as they are."""
    g = torch.zeros(3, 50, device=DEV)
    g[0, 1] = g[2, 3] = 3e38
    before = g.clone()
    out = torch.empty(3, 50, dtype=torch.bfloat16, device=DEV)
    for lst in (training.GradientList([g]), training.GradientList([g], [out])):
        assert float(lst.fira_gradient_norm()) == math.inf
        assert float(lst.fira_clip_gradients(limit)) == math.inf
    assert torch.equal(g, before) and torch.equal(out, before.to(torch.bfloat16))


@pytest.mark.parametrize("limit", [1.0, 1e38])
def test_the_largest_norms_are_cut(limit):
    """Norms just inside the range: the caller reads a finite one, and the gradients are scaled by it."""
    g = torch.zeros(3, 50, device=DEV)
    g[0, 1] = g[2, 3] = 2.4e38
    norm = math.sqrt(2.0) * float(g[0, 1])
    assert abs(float(training.GradientList([g]).fira_clip_gradients(limit)) / norm - 1.0) < 1e-6
    assert abs(float(g[0, 1]) / (limit / math.sqrt(2.0)) - 1.0) < 1e-6 and float(g[1, 1]) == 0.0
