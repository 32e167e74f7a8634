"""AdamW, rotary positions and the block norm together with the operators and the step that were there, as a training run uses them: the example runs, its gradients are
those of torch's own operations in fp64, and its AdamW step is the definition's on those gradients."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import model_reference as ref
from training_reference import HALF_ULP, TINY, f64, within

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_attention_lm.py")


def _example():
    spec = importlib.util.spec_from_file_location("train_attention_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("state", [torch.float32, torch.float8_e4m3fn])
def test_the_example_runs(state):
    model, losses, norms = _example().train(steps=12, state=state)
    assert all(math.isfinite(x) for x in losses + norms) and model.adamw.t.tolist() == [12, 0]
    assert abs(losses[0] - math.log(512)) < 0.5          # it starts by knowing nothing
    assert all(torch.isfinite(p.float()).all() for p in model.p.values())


def _in_64_bits(model, ids):
    """The model in elementary torch operations in fp64 -> (loss, gradients)."""
    p = {k: v.detach().double().requires_grad_(True) for k, v in model.p.items()}
    rms = lambda x, w: x * (x.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w  # noqa: E731
    b, n = ids.shape[0], ids.shape[1] - 1
    h, k, head, half = model.heads, model.kv_heads, model.head, len(model.frequencies)
    angle = torch.arange(n, device=ids.device, dtype=torch.float64)[:, None] * model.frequencies
    c, s = (model.turn_scale * f[:, None] for f in (angle.cos(), angle.sin()))

    def turn(x):
        a, z = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * c - z * s, a * s + z * c, x[..., 2 * half:]], -1)

    x = p["table"][ids[:, :-1]] * model.scale
    qkv = (rms(x, p["norm0"]) @ p["qkv"]).view(b, n, h + 2 * k, head)
    q, key, value = turn(qkv[:, :, :h]), turn(qkv[:, :, h:h + k]).repeat_interleave(h // k, 2), qkv[:, :, h + k:].repeat_interleave(h // k, 2)
    scores = torch.einsum("bihd,bjhd->bhij", q, key) / math.sqrt(head)
    scores = scores.masked_fill(torch.ones(n, n, dtype=torch.bool, device=ids.device).triu(1), -math.inf)
    block = torch.einsum("bhij,bjhd->bihd", scores.softmax(-1), value).reshape(b, n, h * head) @ p["out"]
    x = x + p["gate1"] * rms(block, p["post1"])
    block = torch.nn.functional.silu(rms(x, p["norm1"]) @ p["up"]) @ p["down"]
    x = x + p["gate2"] * rms(block, p["post2"])
    loss = torch.nn.functional.cross_entropy((rms(x, p["norm2"]) @ p["unembed"]).flatten(0, 1), ids[:, 1:].flatten())
    loss.backward()
    return loss, {k: v.grad for k, v in p.items()}


def test_gradients_and_the_step_after_them():
    """bf16 activations on both sides of a bf16 model leave a few roundings of 2^-9 each (relative, in the mean), of which some forty lie between the loss and the
    first norm's weight, in the forward pass and back: sqrt(80) 2^-9 < 2e-2; their products with what they meet, twice that."""
    ex = _example()
    model = ex.AttentionModel(vocab=96, dim=64, heads=4, kv_heads=2, hidden=128, rank=16)
    gen = torch.Generator(device=ex.DEV)
    gen.manual_seed(3)
    for k, v in model.p.items():
        if v.dim() == 1:
            v.add_(0.2 * torch.randn(v.shape, device=ex.DEV, generator=gen))
        else:
            v.mul_(4.0)                                    # so that blocks and scores are of some size
    ids = torch.randint(0, 96, (16, 21), device=ex.DEV, generator=gen)
    for t in model.total.values():
        t.zero_()
    loss = model.loss(ids)
    loss.backward()
    want, grads = _in_64_bits(model, ids)
    loss, want = float(loss.detach()), float(want.detach())
    assert abs(loss - want) < 1e-2 * want
    for k, t in model.total.items():
        assert float((t.double() - grads[k]).norm() / grads[k].norm()) < 4e-2, k

    norm = model.clip.fira_clip_gradients(model.max_norm)
    assert abs(float(norm) / math.sqrt(sum(float(t.double().square().sum()) for t in model.total.values())) - 1) < 1e-6
    params = [(k, model.p[k]) for k in model.p if k not in model.matrices]
    before = {k: (f64(p).reshape(-1), f64(model.grad[k]).reshape(-1)) for k, p in params}
    model.adamw.fira_adamw_step(3e-3, beta2=0.99)
    for k, p in params:
        w, g = before[k]
        x, off = ref.adamw(w, g, np.zeros_like(w), np.zeros_like(w), 0, 0.01 if p.dim() == 2 else 0.0, 3e-3, 0.9, 0.99, 1e-8)["w"]
        within(p.reshape(-1), x, off + HALF_ULP[p.dtype] * (np.abs(x) + off) * (1 + 1e-3) + TINY)
