"""AdamW's ways through its kernels, each against the definition in 64 bits (tests/model_reference.py): lists without rows that are apart, of more than a tile; rows apart
and whole vectors wide, or not, with and without results at whole lines; tensors and states cut from one buffer at any element or byte, with what lies between left
as it was; pieces that begin inside a row."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01623_amd import training

import model_reference as ref
import test_gpu_adamw as base
from test_gpu_adamw import BF16, E4M3, F32, HYPER, TYPES
from training_reference import HALF_ULP, TINY, U, f64, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def steps(params, gs, decays, lst, gen, count=3):
    for k in range(count):
        before = base.Snapshot(lst, params, gs)
        lst.fira_adamw_step(1e-2, **HYPER)
        base.check(lst, params, before, decays, 1e-2)
        for g in gs:
            g.copy_((1e-3 * (3.0 if k == 1 else 1.0) * torch.randn(g.shape, device=DEV, generator=gen)).to(g.dtype))


# (a tile has up to 4096 values)
DENSE = [((1, 1), 0), ((1, 4095), 0), ((1, 4096), 0), ((3, 4097), 0), ((7, 1000), 0), ((1, 100003), 0), ((64, 520), 0), ((1, 257), 0), ((2, 2048), 0)]
WHOLE_VECTORS = [((40, 520), 8), ((33, 1000), 24), ((5, 4096), 64), ((300, 8), 8), ((70, 72), 56), ((2, 16), 48), ((1, 5000), 0), ((130, 64), 0)]
ODD = [((33, 1001), 23), ((9, 4097), 63), ((100, 3), 61), ((400, 127), 1), ((40, 520), 8), ((17, 2050), 0), ((1, 10000), 0)]


@pytest.mark.parametrize("shapes", [DENSE, WHOLE_VECTORS, ODD], ids=["dense", "whole_vectors", "odd"])
@pytest.mark.parametrize("state", [F32, E4M3])
@pytest.mark.parametrize("dtype,grads", TYPES)
def test_lists(dtype, grads, state, shapes):
    """Rows apart of `odd` and `whole_vectors` begin at whole lines of 128 bytes in bf16 or in fp32 for some, and not for others."""
    bufs, params, gbufs, gs, decays, lst, gen = base.problem(dtype, grads, state, 21, shapes)
    steps(params, gs, decays, lst, gen)
    for (shape, _), b in zip(shapes, bufs):
        assert torch.isnan(b[:, shape[1]:].float()).all()


def cut(sizes, first, dtype, gen, scale):
    """Pieces of one buffer, one after the other, the first from element `first` on, and the buffer's parts before and behind."""
    n = sum(sizes)
    flat = torch.full((first + n + 100,), 7, dtype=torch.uint8, device=DEV).view(dtype) if dtype is E4M3 else torch.full((first + n + 100,), 7.0, dtype=dtype, device=DEV)
    if scale:
        flat[first:first + n] = (scale * torch.randn(n, device=DEV, generator=gen)).to(dtype)
    elif dtype is E4M3:
        flat.view(torch.uint8)[first:first + n] = 0
    else:
        flat[first:first + n] = 0.0
    pieces, at = [], first
    for size in sizes:
        pieces.append(flat[at:at + size])
        at += size
    return pieces, flat[:first].view(torch.uint8) if dtype is E4M3 else flat[:first], flat[at:].view(torch.uint8) if dtype is E4M3 else flat[at:]


@pytest.mark.parametrize("first", [1, 3, 64, 67])
@pytest.mark.parametrize("state", [F32, E4M3])
@pytest.mark.parametrize("dtype,grads", TYPES)
def test_tensors_cut_from_one_buffer(dtype, grads, state, first):
    """As trainers keep them: neighbours without a gap, at odd elements, their codes at odd bytes."""
    gen = base.generator(first)
    shapes = [(3, 4097), (1, 5), (20, 1000), (1, 255), (7, 8192), (1, 1), (5, 3333)]
    sizes = [a * b for a, b in shapes]
    blocks = [-(-n // 256) for n in sizes]
    edges, parts = [], {}
    for name, dt, scale, of in (("w", dtype, 0.02, sizes), ("g", grads, 1e-3, sizes), ("m", state, 0.0, sizes), ("v", state, 0.0, sizes), ("ms", F32, 0.0, blocks), ("vs", F32, 0.0, blocks)):
        parts[name], before, behind = cut(of, first, dt, gen, scale)
        edges += [before, behind]
    params, gs = ([x.view(s) for x, s in zip(parts[k], shapes)] for k in "wg")
    decays = [0.1 * (i % 3) for i in range(len(shapes))]
    scales = {} if state is F32 else dict(m_scale=parts["ms"], v_scale=parts["vs"])
    lst = training.AdamWList(params, gs, weight_decay=decays, m=parts["m"], v=parts["v"], **scales)
    steps(params, gs, decays, lst, gen)
    assert all(bool((e == 7).all()) for e in edges)


@pytest.mark.parametrize("state", [F32, E4M3])
def test_a_piece_that_begins_inside_a_row(state):
    """2^30 + 7.7e6 values with rows apart: those around 2^30, where the second piece begins, and the last ones."""
    rows, cols, pad = 33000, 32771, 3
    w, g = (torch.zeros(rows, cols + pad, dtype=BF16, device=DEV)[:, :cols] for _ in range(2))
    gen = base.generator(22)
    parts = [slice(32760, 32770), slice(rows - 2, rows)]
    assert 32761 * cols < 1 << 30 < 32769 * cols
    for at in parts:
        w[at] = (0.02 * torch.randn(w[at].shape, device=DEV, generator=gen)).to(BF16)
        g[at] = (1e-3 * torch.randn(w[at].shape, device=DEV, generator=gen)).to(BF16)
    old = [(f64(w[at]).reshape(-1), f64(g[at]).reshape(-1)) for at in parts]
    lst = training.AdamWList([w], [g], weight_decay=0.1, state=state, seeds=[5])
    lst.fira_adamw_step(1e-2, **HYPER)
    for at, (w0, g0) in zip(parts, old):
        first, n = at.start * cols, len(w0)
        want = ref.adamw(w0, g0, np.zeros(n), np.zeros(n), 0, 0.1, 1e-2, 0.9, 0.999, 1e-8)
        x, off = want["w"]
        within(w[at].reshape(-1), x, off + HALF_ULP[BF16] * (np.abs(x) + off) * (1 + 1e-3) + TINY)
        if state is F32:
            within(lst.m[0][first:first + n], *want["m"])
            within(lst.v[0][first:first + n], *want["v"])
            continue
        # (whole blocks only: what shares a block with the first and last values here is zero)
        random = ref.rounding(n, 5, 1, first=first)
        for codes, scales, (x, _), r, floor in ((lst.m[0], lst.m_scale[0], want["m"], random[0], False), (lst.v[0], lst.v_scale[0], want["root"], random[1], True)):
            shift = first % 256
            most, blocks = ref.block_most(np.concatenate([np.zeros(shift), x]))
            within(scales[first // 256:first // 256 + len(blocks)], blocks / 448.0, 16 * U * blocks / 448.0 + 1e-44)
            got = np.abs(ref.e4m3(codes[first:first + n]))
            low, high = (ref.held(x, most[shift:], r, floor, e * U) for e in (-32, 32))
            assert np.mean((got >= low) & (got <= high)) > 0.9999
    for at in (slice(0, 50), slice(16000, 16050), slice(32700, 32760), slice(32770, 32800)):
        assert not w[at].any() and not lst.m[0][at.start * cols:at.stop * cols].view(torch.uint8).any()


def test_blocks_of_small_values():
    """Scales and codes of blocks whose largest root is 2^-100 and more, which are held, and less, which are not.  With betas of zero m is g and the root |g|, but for roundings of the
    square, the root, the scale and the quotient."""
    exponents = [-99.9, -99.5, -99.0, -98.0, -97.0, -96.0, -95.5, -95.0, -94.0, -93.0, -90.0, -60.0, 0.0, 26.0, 28.0, 31.0, 33.0, 60.0]
    gen = base.generator(23)
    g = 1.0 - 0.4 * torch.rand(len(exponents), 256, device=DEV, generator=gen).double()
    g[:, 7] = 1.0                                          # the largest
    g = (g * torch.tensor([2.0 ** e for e in exponents], dtype=torch.float64, device=DEV)[:, None] * torch.where(torch.rand(256, device=DEV, generator=gen) < 0.5, -1.0, 1.0)).float()
    w = torch.zeros_like(g)
    lst = training.AdamWList([w], [g], state=E4M3, seeds=[3])
    lst.fira_adamw_step(1e-3, beta1=0.0, beta2=0.0, eps=1e-38)
    x = f64(g).reshape(-1)
    random = ref.rounding(len(x), 3, 1)
    # (below 2^-100, which no value but those of the first two blocks is, a root may be held as less)
    fine = np.abs(x) >= 2.0 ** -100
    assert fine[512:].all()
    for codes, scales, r, floor in ((lst.m[0], lst.m_scale[0], random[0], False), (lst.v[0], lst.v_scale[0], random[1], True)):
        most, blocks = ref.block_most(x)
        within(scales, blocks / 448.0, 8 * U * blocks / 448.0)
        got = np.abs(ref.e4m3(codes))
        low, high = (ref.held(x, most, r, floor, e * U) for e in (-8, 8))
        assert np.all(((got >= low) & (got <= high))[fine]) and np.all(got <= high)
    # every step is lr in size
    assert np.all(np.abs(np.abs(f64(w)).reshape(-1) - 1e-3)[fine] <= 16 * U * 1e-3)
    lst = training.AdamWList([torch.zeros(1, 256, device=DEV)], [g[:1] * 0.9], state=E4M3)
    lst.fira_adamw_step(1e-3, beta1=0.0, beta2=0.0)
    assert not any(bool(t.float().any()) for t in (lst.m[0], lst.v[0], lst.m_scale[0], lst.v_scale[0]))       # (zeros of either sign)


def test_scales_and_codes_are_the_headers():
    """With betas of zero, m is g and the root |g| (of a square that is rounded, the rounded root is what was squared).  The scale is the largest size times fp32's 1/448, and what a code is
    of the value times ((1 / largest) times 448), each rounded: the same bits for blocks of every size in fp32's range."""
    one = np.float32
    blocks = 4096
    gen = base.generator(24)
    size = torch.exp2(torch.linspace(-80.0, 61.0, blocks, device=DEV))[:, None]
    g = size * torch.randn(blocks, 256, device=DEV, generator=gen)
    lst = training.AdamWList([torch.zeros(blocks, 256, device=DEV)], [g], state=E4M3, seeds=[9])
    lst.fira_adamw_step(1e-3, beta1=0.0, beta2=0.0)
    x = g.cpu().numpy()
    most = np.abs(x).max(1)
    factor = (one(1.0) / most) * one(448.0)
    y = np.minimum(np.abs(x) * factor[:, None], one(448.0)).reshape(-1).astype(np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3.0)
    random = ref.rounding(x.size, 9, 1)
    plain = y >= 2.0 ** -6                                 # (smaller sizes are added to 2^-6 before they are rounded, in fp32)
    for codes, scales, r in ((lst.m[0], lst.m_scale[0], random[0]), (lst.v[0], lst.v_scale[0], random[1])):
        assert np.array_equal(scales.cpu().numpy(), most * (one(1.0) / one(448.0)))
        c = np.minimum(np.floor(y / step + (r.astype(np.float64) + 0.5) / 65536.0) * step, 448.0)
        assert np.array_equal(np.abs(ref.e4m3(codes))[plain], c[plain])


@pytest.mark.parametrize("state", [F32, E4M3])
def test_one_buffer_for_two_states_is_refused(state):
    """m of one tensor that is v of another, scales that are listed twice."""
    from paper_2410_01623_amd import fira
    p, g = [torch.zeros(2, 256, device=DEV) for _ in range(2)], [torch.zeros(2, 256, device=DEV) for _ in range(2)]
    held = lambda: [torch.zeros(512, dtype=torch.uint8, device=DEV).view(E4M3) if state is E4M3 else torch.zeros(512, device=DEV) for _ in range(2)]  # noqa: E731
    scale = lambda: [torch.zeros(2, device=DEV) for _ in range(2)]  # noqa: E731
    m, v, ms, vs = held(), held(), scale(), scale()
    scales = dict(m_scale=ms, v_scale=vs) if state is E4M3 else {}
    training.AdamWList(p, g, m=m, v=v, **scales)
    bad = [dict(m=m, v=[v[0], m[0]], **scales)]
    if state is E4M3:
        bad += [dict(m=m, v=v, m_scale=[ms[0], ms[0]], v_scale=vs), dict(m=m, v=v, m_scale=ms, v_scale=[vs[0], ms[0]]), dict(m=m, v=v, m_scale=ms, v_scale=ms)]
    for kw in bad:
        with pytest.raises(fira.FiraError, match="twice"):
            training.AdamWList(p, g, **kw)
