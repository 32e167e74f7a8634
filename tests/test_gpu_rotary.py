"""Rotary positions and their gradient against the definition in 64 bits (tests/model_reference.py), where they can go wrong: heads of two values and odd
ones, parts that are not turned, parts of one buffer with NaN around them, permuted and expanded tensors, results in place, far and negative positions, one
token, none, offsets beyond 32 bits, graphs and streams."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01623_amd import fira, training

import model_reference as ref
from training_reference import U, f64, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
CALLS = [training.fira_rotary, training.fira_rotary_gradient]
# batch, length, heads, key heads, dim, rotated
SHAPES = [(1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (3, 5, 4, 2, 64, 64), (2, 7, 3, 1, 64, 32), (1, 33, 5, 5, 80, 80), (2, 9, 2, 1, 96, 72), (1, 4, 7, 3, 17, 6), (2, 3, 2, 2, 20, 20),
          (1, 300, 6, 2, 40, 24), (4, 65, 9, 1, 256, 256), (1, 2, 1, 1, 515, 514), (2, 130, 1, 1, 33, 32), (1, 17, 40, 4, 192, 64), (1, 3, 2, 1, 16384, 16384)]


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def check(call, got, x, positions, f, interleaved, scale):
    """positions: (batch, length), on the host."""
    shape = (-1, *x.shape[-3:])
    within(got.reshape(shape), *ref.rotary(x.reshape(shape), positions, f, interleaved, scale, call is training.fira_rotary_gradient))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,length,heads,kv_heads,dim,rotated", SHAPES)
def test_shapes(batch, length, heads, kv_heads, dim, rotated, dtype, interleaved):
    """Queries and keys as parts of one buffer whose other values are NaN, into parts of another; positions counted, of each sequence, and shared."""
    gen = generator(dim + length)
    f, _ = training.fira_rotary_frequencies(rotated)
    for pad in (0, 3):
        buffers = [torch.full((batch, length, heads + 2 * kv_heads, dim + pad), math.nan, dtype=dtype, device=DEV) for _ in range(2)]
        (q, k), (qo, ko) = ([b[:, :, :heads, :dim], b[:, :, heads:heads + kv_heads, :dim]] for b in buffers)
        for x in (q, k):
            x.copy_(torch.randn(x.shape, device=DEV, generator=gen).to(dtype))
        counted = np.arange(length)[None].repeat(batch, 0)
        own = torch.randint(-5, 5000, (batch, length), device=DEV, generator=gen)
        for positions, where in ((None, counted), (own.to(torch.int32), own.cpu().numpy()), (own[0].contiguous(), own[:1].cpu().numpy().repeat(batch, 0))):
            for call in CALLS:
                got = call(q, k, positions, f, interleaved=interleaved, scale=1.3, q_out=qo, k_out=ko)
                assert got[0] is qo and got[1] is ko
                check(call, qo, q, where, f, interleaved, 1.3)
                check(call, ko, k, where, f, interleaved, 1.3)
                assert torch.isnan(buffers[1][:, :, heads + kv_heads:].float()).all() and torch.isnan(buffers[1][..., dim:].float()).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,rotated", [(50, 50), (98, 98), (130, 130), (130, 26), (256, 254), (64, 10), (72, 18), (27, 16), (35, 34), (254, 254), (1030, 1026)])
def test_heads_that_are_no_whole_vectors(dim, rotated, dtype, interleaved):
    """Vectors overlap at the end of a half and of what is copied: many heads and tokens, more than a workgroup has, into other tensors and in place; the same bits both ways."""
    gen = generator(dim + rotated)
    f, _ = training.fira_rotary_frequencies(rotated)
    for tokens, heads in ((3, 5), (700, 9)):
        q, k = (torch.randn(2, tokens, h, dim, device=DEV, generator=gen).to(dtype) for h in (heads, 2))
        where = np.arange(tokens)[None].repeat(2, 0)
        for call in CALLS:
            got = call(q, k, None, f, interleaved=interleaved, scale=0.9)
            check(call, got[0], q, where, f, interleaved, 0.9)
            check(call, got[1], k, where, f, interleaved, 0.9)
            for _ in range(3):
                a, b = q.clone(), k.clone()
                call(a, b, None, f, interleaved=interleaved, scale=0.9, q_out=a, k_out=b)
                assert torch.equal(a, got[0]) and torch.equal(b, got[1])
            a, b = q.clone(), torch.empty_like(k)
            call(a, k, None, f, interleaved=interleaved, scale=0.9, q_out=a, k_out=b)
            assert torch.equal(a, got[0]) and torch.equal(b, got[1])


@pytest.mark.parametrize("far", [10 ** 6, (1 << 31) - 5, 1 << 36, -10 ** 7])
def test_far_positions(far):
    gen = generator(1)
    f, _ = training.fira_rotary_frequencies(128)
    q, k = (torch.randn(1, 9, h, 128, device=DEV, generator=gen) for h in (3, 1))
    positions = far + torch.arange(9, device=DEV)[None]
    for call in CALLS:
        got = call(q, k, positions, f)
        check(call, got[0], q, positions.cpu().numpy(), f, False, 1.0)
        check(call, got[1], k, positions.cpu().numpy(), f, False, 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views(dtype, interleaved):
    """Heads before tokens, one head for all, sequences in two dimensions, no dimension of sequences, and what has no such strides; alone and in place."""
    gen = generator(2)
    f, _ = training.fira_rotary_frequencies(48)
    base = torch.randn(2, 6, 10, 64, device=DEV, generator=gen).to(dtype)
    views = [base.transpose(1, 2), base[:, :, :1].expand(2, 6, 10, 64), base.view(2, 2, 3, 10, 64), base[0], base[::2, ::3], base.permute(0, 3, 1, 2)[..., :6].transpose(-1, -2)[..., :6, :].transpose(-1, -2),
             torch.randn(2, 3, 50, 64, device=DEV, generator=gen).to(dtype).transpose(-1, -3)[:, :, :, :3].transpose(-1, -3)]
    views = [v if v.shape[-1] >= 48 else torch.randn(2, 5, 4, 128, device=DEV, generator=gen).to(dtype)[..., ::2] for v in views]
    for x in views:
        batch, length = math.prod(x.shape[:-3]), x.shape[-3]
        where = np.arange(length)[None].repeat(batch, 0)
        got, none = training.fira_rotary(x, None, None, f, interleaved=interleaved)
        assert none is None and got.shape == x.shape
        check(training.fira_rotary, got, x, where, f, interleaved, 1.0)
    for x in (base, base.transpose(1, 2), base[:, :, 3:7]):
        old = x.clone()
        want, _ = training.fira_rotary(old, None, None, f, interleaved=interleaved)
        got, _ = training.fira_rotary(x, None, None, f, interleaved=interleaved, q_out=x)
        assert got is x and torch.equal(x, want)


def test_the_gradient_is_the_transpose():
    """<dy, turn(x)> = <gradient(dy), x>, and turning back by the gradient gives scale^2 x."""
    gen = generator(3)
    f, scale = training.fira_rotary_frequencies(64, context=fira.FIRA_ROTARY_BY_PARTS, factor=8.0)
    x, dy = torch.randn(2, 50, 4, 96, device=DEV, generator=gen), torch.randn(2, 50, 4, 96, device=DEV, generator=gen)
    y, _ = training.fira_rotary(x, None, None, f, scale=scale)
    dx, _ = training.fira_rotary_gradient(dy, None, None, f, scale=scale)
    a, b = (y.double() * dy.double()), (dx.double() * x.double())
    assert abs(float(a.sum() - b.sum())) <= 40 * U * scale * float((x.double().abs() * dy.double().abs()).sum() * 2)
    back, _ = training.fira_rotary_gradient(y, None, None, f, scale=scale)
    want = x.double() * torch.where(torch.arange(96, device=DEV) < 64, scale * scale, 1.0)
    assert float((back.double() - want).abs().max()) <= 60 * U * float(x.abs().max()) * 2 * scale * scale
    # along a direction, a difference is the gradient's product with it (the turn is linear)
    v = torch.randn(x.shape, device=DEV, generator=gen)
    ends = [float((training.fira_rotary(x + e * v, None, None, f, scale=scale)[0].double() * dy.double()).sum()) for e in (0.5, -0.5)]
    along = (dx.double() * v.double())
    assert abs(ends[0] - ends[1] - float(along.sum())) <= 1e-4 * float(along.square().sum().sqrt())


def test_frequencies():
    j = np.arange(32)
    plain = 10000.0 ** (-j / 32)
    f, scale = training.fira_rotary_frequencies(64)
    assert scale == 1.0 and f.dtype == torch.float64 and f.device.type == "cuda" and np.abs(f64(f) / plain - 1).max() < 1e-14
    f, scale = training.fira_rotary_frequencies(64, context=fira.FIRA_ROTARY_LINEAR, factor=4.0)
    assert scale == 1.0 and np.abs(f64(f) / (plain / 4) - 1).max() < 1e-14
    f, scale = training.fira_rotary_frequencies(64, 500000.0, context=fira.FIRA_ROTARY_BY_PARTS, factor=16.0, trained=8192.0, low=2.0, high=20.0)
    plain = 500000.0 ** (-j / 32)
    keep = np.clip((8192.0 * plain / (2 * math.pi) - 2.0) / 18.0, 0, 1)
    assert abs(scale - (0.1 * math.log(16.0) + 1)) < 1e-15 and np.abs(f64(f) / (plain * keep + plain / 16 * (1 - keep)) - 1).max() < 1e-13
    assert (keep == 1).any() and (keep == 0).any() and ((keep > 0) & (keep < 1)).any()


def test_no_tokens_and_no_heads():
    f, _ = training.fira_rotary_frequencies(8)
    for shape in ((0, 3, 2, 8), (2, 0, 2, 8), (2, 3, 0, 8)):
        got, k = training.fira_rotary(torch.empty(shape, device=DEV), torch.empty(shape, device=DEV), None, f)
        assert got.shape == shape and k.shape == shape


def test_refusals():
    f, _ = training.fira_rotary_frequencies(8)
    q, k = torch.zeros(2, 3, 4, 16, device=DEV), torch.zeros(2, 3, 2, 16, device=DEV)
    ids = torch.zeros(2, 3, dtype=torch.int64, device=DEV)
    bad = [(q[0, 0], None, None, f, {}), (q, k[:1], None, f, {}), (q, k[..., :8], None, f, {}), (q, k.to(BF16), None, f, {}), (q.half(), None, None, f, {}), (q, k, ids.float(), f, {}),
           (q, k, ids[:, :2], f, {}), (q, k, None, f.float(), {}), (q, k, None, f[:, None], {}), (q, k, None, f.repeat(3), {}), (q, k, None, f[:0], {}), (q, k.cpu(), None, f, {}),
           (q, k, None, f, dict(q_out=k)), (q, None, None, f, dict(k_out=k)), (q, k, None, f, dict(scale=math.inf)), (q, k, None, f, dict(q_out=q[:, :, :1].expand(2, 3, 4, 16))),
           (q, k, None, f, dict(q_out=torch.zeros(2, 3, 4, 32, device=DEV)[..., ::2]))]
    for a, b, p, fr, kw in bad:
        with pytest.raises(fira.FiraError):
            training.fira_rotary(a, b, p, fr, **kw)
    with pytest.raises(fira.FiraError):                     # in place with other strides
        training.fira_rotary(q.transpose(1, 2), None, None, f, q_out=q.view(2, 4, 3, 16))


def test_beyond_32_bit_offsets():
    tokens, heads, dim = 70001, 256, 128                   # 2.3e9 values
    f, _ = training.fira_rotary_frequencies(dim)
    q = torch.zeros(1, tokens, heads, dim, dtype=BF16, device=DEV)
    q[0, -2:].normal_(generator=generator(4))
    last = q[:, -2:].clone()
    training.fira_rotary(q, None, None, f, q_out=q)
    check(training.fira_rotary, q[:, -2:], last, np.array([[tokens - 2, tokens - 1]]), f, False, 1.0)
    assert not q[0, :100].any() and not q[0, tokens // 2].any() and not q[0, -100:-2].any()


def test_in_a_graph_and_on_a_stream(no_automatic_collection):
    gen = generator(5)
    f, _ = training.fira_rotary_frequencies(64)
    q, k = (torch.randn(2, 33, h, 64, device=DEV, generator=gen).to(BF16) for h in (8, 2))
    positions = torch.zeros(2, 33, dtype=torch.int64, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = training.fira_rotary(q, k, positions, f)
        back = training.fira_rotary_gradient(got[0], got[1], positions, f)
    for step in range(4):
        q.normal_(generator=gen)
        k.normal_(generator=gen)
        positions.copy_(torch.randint(0, 10000, positions.shape, device=DEV, generator=gen))
        graph.replay()
        want = training.fira_rotary(q, k, positions, f)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(back[0], training.fira_rotary_gradient(*want, positions, f)[0])
    torch.cuda.synchronize()
    other = training.fira_rotary(q, k, positions, f, stream=side)
    side.synchronize()
    assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])
    del graph
