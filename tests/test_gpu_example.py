"""The example's model learns its language: all operators around the step and the step itself, together."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_small_lm.py")


def _example():
    spec = importlib.util.spec_from_file_location("train_small_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_small_model_learns():
    losses, norms = _example().train(steps=80)
    assert all(math.isfinite(x) for x in losses + norms)
    assert abs(losses[0] - math.log(768)) < 0.5          # it starts by knowing nothing
    assert losses[-1] < 0.5 * losses[0]


def test_gradients_of_the_example_are_autograds():
    """The example's gradients against torch's own modules in fp32, differentiated by autograd; bf16 activations on both sides of a
    bf16 model leave a few roundings of 2^-8 each."""
    import torch
    ex = _example()
    model = ex.SmallModel(vocab=96, dim=64, hidden=128, rank=16)
    gen = torch.Generator(device=ex.DEV)
    gen.manual_seed(3)
    model.p["ln_w"].add_(0.2 * torch.randn(1, 64, device=ex.DEV, generator=gen))
    model.p["ln_b"].add_(0.2 * torch.randn(1, 64, device=ex.DEV, generator=gen))
    ids = torch.randint(0, 96, (16, 21), device=ex.DEV, generator=gen)
    for t in model.total.values():
        t.zero_()
    loss = model.loss(ids)
    loss.backward()
    p = {k: v.detach().double().requires_grad_(True) for k, v in model.p.items()}
    x = p["table"][ids[:, :-1]] * model.scale
    n = torch.nn.functional.layer_norm(x, (64,), p["ln_w"][0], p["ln_b"][0])
    h = x + torch.nn.functional.silu(n @ p["up"]) @ p["down"]
    r = h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * p["rms_w"][0]
    want = torch.nn.functional.cross_entropy((r @ p["head"]).flatten(0, 1), ids[:, 1:].flatten())
    want.backward()
    assert abs(float(loss) - float(want)) < 1e-2 * float(want)
    for k, t in model.total.items():
        ref = p[k].grad
        assert float((t.double() - ref).norm() / ref.norm()) < 3e-2, k
