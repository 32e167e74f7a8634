"""AdamW over lists of tensors against its definition in 64 bits (tests/model_reference.py), where it can go wrong: tensors of one value, ends of
blocks, rows apart with NaN in between, all pairs of types, states in both forms, gradients that are cut, the first step and late ones, values that are not
finite, learning rates on the GPU, graphs, streams, offsets beyond 32 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01623_amd import fira, training

import model_reference as ref
from training_reference import HALF_ULP, TINY, U, f64, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
TYPES = [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)]
SHAPES = [((1, 1), 0), ((1, 255), 0), ((1, 256), 0), ((1, 257), 0), ((3, 7), 2), ((5, 300), 3), ((300, 5), 1), ((2, 8), 8), ((129, 72), 0), ((40, 520), 8), ((3, 33333), 0), ((70, 1), 3)]
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def matrix(shape, pad, dtype, gen, scale):
    rows, cols = shape
    buf = torch.full((rows, cols + pad), math.nan, dtype=dtype, device=DEV)
    buf[:, :cols] = (scale * torch.randn(rows, cols, device=DEV, generator=gen)).to(dtype)
    return buf, buf[:, :cols]


def same(a, b):
    return all(torch.equal(x.reshape(-1).view(torch.uint8), y.reshape(-1).view(torch.uint8)) for x, y in zip(a, b))


class Snapshot:
    """What a step starts from."""

    def __init__(self, lst, params, grads):
        self.taken = int(lst.t[0])
        self.w, self.g = [f64(p).reshape(-1) for p in params], [f64(g).reshape(-1) for g in grads]
        self.m, self.v = [], []
        for i in range(lst.count):
            if lst.m_scale[i] is None:
                self.m.append(f64(lst.m[i]))
                self.v.append(f64(lst.v[i]))
            else:
                place = np.arange(lst.m[i].numel()) // 256
                m, root = (np.float32(ref.e4m3(c)) * s.cpu().numpy()[place] for c, s in ((lst.m[i], lst.m_scale[i]), (lst.v[i], lst.v_scale[i])))
                self.m.append(m.astype(np.float64))
                self.v.append((root * root).astype(np.float64))


def check(lst, params, before, decays, lr, cut=1.0, seeds=None):
    assert int(lst.t[0]) == before.taken + 1 and int(lst.t[1]) == 0
    for i, p in enumerate(params):
        if not p.numel():
            continue
        want = ref.adamw(before.w[i], before.g[i], before.m[i], before.v[i], before.taken, decays[i], lr, HYPER["beta1"], HYPER["beta2"], HYPER["eps"], cut)
        w, off = want["w"]
        within(p.reshape(-1), w, off + HALF_ULP[p.dtype] * (np.abs(w) + off) * (1 + 1e-3) + TINY)
        if lst.m_scale[i] is None:
            within(lst.m[i], *want["m"])
            within(lst.v[i], *want["v"])
            continue
        random = ref.rounding(p.numel(), i if seeds is None else seeds[i], before.taken + 1)
        for codes, scales, (x, off), r, floor in ((lst.m[i], lst.m_scale[i], want["m"], random[0], False), (lst.v[i], lst.v_scale[i], want["root"], random[1], True)):
            most, blocks = ref.block_most(x)
            off_most = np.pad(np.where(np.isfinite(off), off, 0.0), (0, -len(off) % 256)).reshape(-1, 256).max(1)
            within(scales, blocks / 448.0, off_most / 448.0 + 2 * U * blocks / 448.0 + 1e-44)
            # the code of a value is that of one within its error: x is off by `off`, the largest one by off_most, the quotient by three roundings
            with np.errstate(invalid="ignore", divide="ignore"):
                slack = np.where(x != 0.0, off / np.abs(x), 0.0) + np.repeat(off_most / np.maximum(blocks, 1e-300), 256)[:len(x)] + 4 * U
            got = ref.e4m3(codes)
            low, high = (ref.held(x, most, r, floor, e) for e in (-slack, slack))
            bad = np.isnan(low)
            assert np.array_equal(np.isnan(got), bad)
            inside = (np.abs(got) >= low) & (np.abs(got) <= high)
            # (a size below 2^-6 loses what is under 2^-30 when it is added to that: a 2^-21st of a step, which is rarely between it and its number)
            small = np.abs(x) * 448.0 / np.maximum(most, 1e-300) < 2.0 ** -6
            assert np.all((inside | small)[~bad]) and (~inside & ~bad).sum() <= 2 + len(x) // 100000
            assert np.all((np.sign(got) * np.sign(x) >= 0) | bad)


def problem(dtype, grads, state, seed, shapes=SHAPES, scale=1e-3):
    gen = generator(seed)
    bufs, params, gbufs, gs = [], [], [], []
    for shape, pad in shapes:
        b, p = matrix(shape, pad, dtype, gen, 0.02)
        c, g = matrix(shape, pad if len(params) % 2 else 0, grads, gen, scale)
        bufs.append(b), params.append(p), gbufs.append(c), gs.append(g)
    decays = [0.1 * (i % 3) for i in range(len(params))]
    return bufs, params, gbufs, gs, decays, training.AdamWList(params, gs, weight_decay=decays, state=state), gen


@pytest.mark.parametrize("state", [F32, E4M3])
@pytest.mark.parametrize("dtype,grads", TYPES)
def test_steps(dtype, grads, state):
    bufs, params, gbufs, gs, decays, lst, gen = problem(dtype, grads, state, 1)
    for k in range(4):
        before = Snapshot(lst, params, gs)
        lst.fira_adamw_step(1e-2, **HYPER)
        check(lst, params, before, decays, 1e-2)
        for (shape, _), b, c, g in zip(SHAPES, bufs, gbufs, gs):
            assert torch.isnan(b[:, shape[1]:].float()).all() and torch.isnan(c[:, shape[1]:].float()).all()
            g.copy_((1e-3 * (3.0 if k == 1 else 1.0) * torch.randn(shape, device=DEV, generator=gen)).to(grads))


def test_codes_are_those_of_elementary_operations():
    """In 8 bits, too, every product, sum, root and quotient is rounded to nearest by itself, but for one in millions; and a value that is off by an ulp has another code by one chance in
    2^17 (2^20 ulp to a step, of which a code takes its part down to 2^3).  So 50000 values have the same codes and scales as in numpy, step after step."""
    one = np.float32
    _, params, _, gs, _, lst, gen = problem(BF16, F32, E4M3, 8, [((50, 1000), 0)])
    m, v = np.zeros(50000, one), np.zeros(50000, one)
    place = np.arange(50000) // 256
    for k in range(4):
        lst.fira_adamw_step(1e-3, **HYPER)
        g = gs[0].cpu().numpy().reshape(-1)
        m = m * one(0.9) + g * one(1.0 - 0.9)
        v = v * one(0.999) + g * g * one(1.0 - 0.999)
        random = ref.rounding(50000, 0, k + 1)
        held = []
        for x, r, codes, scales in ((m, random[0], lst.m[0], lst.m_scale[0]), (np.sqrt(v), random[1], lst.v[0], lst.v_scale[0])):
            most = np.pad(np.abs(x), (0, -len(x) % 256)).reshape(-1, 256).max(1)
            scale = most * (one(1.0) / one(448.0))
            y = np.minimum(np.abs(x) * (one(1.0) / most * one(448.0))[place], one(448.0)).astype(np.float64)
            step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3.0)
            c = np.minimum(np.floor(y / step + (r.astype(np.float64) + 0.5) / 65536.0) * step, 448.0)
            c = np.copysign(np.where(x > 0, np.maximum(c, 2.0 ** -9), c) if codes is lst.v[0] else c, x)
            # (sizes below 2^-6 are added to that before they are rounded, in fp32)
            got, plain = ref.e4m3(codes), y >= 2.0 ** -6
            assert np.array_equal(got[plain], c[plain]) and (got != c).sum() <= 2
            assert np.array_equal(scales.cpu().numpy(), scale)
            held.append(got.astype(one) * scale[place])
        m, v = held[0], held[1] * held[1]
        gs[0].copy_(1e-3 * (k + 1) * torch.randn(50, 1000, device=DEV, generator=gen))


@pytest.mark.parametrize("taken", [0, 9, 1000, 10 ** 6, (1 << 32) + 5])
def test_step_counts(taken):
    for state in (F32, E4M3):
        _, params, _, gs, decays, lst, _ = problem(BF16, F32, state, 2, SHAPES[4:8])
        lst.fira_adamw_step(1e-3, **HYPER)
        lst.t[0] = taken
        before = Snapshot(lst, params, gs)
        lst.fira_adamw_step(1e-3, **HYPER)
        check(lst, params, before, decays, 1e-3)


@pytest.mark.parametrize("state", [F32, E4M3])
@pytest.mark.parametrize("share", [0.25, 2.0, math.inf])
def test_cut_by_the_norm(share, state):
    """The norm that a list of the same gradients measures; above the limit the step is that of gradients times max_norm / norm, below it of the gradients."""
    _, params, _, gs, decays, lst, _ = problem(BF16, BF16, state, 3)
    norm = training.GradientList(gs).fira_gradient_norm()
    limit = share * float(norm)
    before = Snapshot(lst, params, gs)
    lst.fira_adamw_step(1e-2, **HYPER, norm=norm, max_norm=limit)
    check(lst, params, before, decays, 1e-2, min(1.0, limit / float(norm)))


@pytest.mark.parametrize("norm,max_norm,cut", [(math.inf, 1.0, 1.0), (math.nan, 1.0, 1.0), (0.0, 1.0, 1.0), (0.0, 0.0, 1.0), (3.0, 0.0, 0.0), (2.0, 2.0, 1.0)])
def test_norms_that_cut_nothing_or_all(norm, max_norm, cut):
    _, params, _, gs, decays, lst, _ = problem(F32, BF16, F32, 4, SHAPES[4:7])
    lst.fira_adamw_step(1e-2, **HYPER)
    before = Snapshot(lst, params, gs)
    lst.fira_adamw_step(1e-2, **HYPER, norm=torch.tensor(norm, device=DEV), max_norm=max_norm)
    check(lst, params, before, decays, 1e-2, cut)


@pytest.mark.parametrize("state", [F32, E4M3])
def test_learning_rate_on_the_gpu(state):
    runs = []
    for lr in (3e-3, torch.tensor(3e-3, device=DEV)):
        _, params, _, _, _, lst, _ = problem(BF16, F32, state, 5)
        lst.fira_adamw_step(float(np.float32(3e-3)) if isinstance(lr, float) else lr, **HYPER)
        runs.append([p.clone() for p in params] + lst.m + lst.v)
    assert same(*runs)


@pytest.mark.parametrize("state", [F32, E4M3])
def test_a_tensor_does_not_depend_on_the_list(state):
    """Alone, in the whole list, and in one of 150 tensors; with rows apart and without; and the same call gives the same bits."""
    gen = generator(6)
    w0, g = (x * torch.randn(41, 1043, device=DEV, generator=gen) for x in (0.02, 1e-3))
    results = []
    for pad, others in ((0, 0), (0, 11), (5, 0), (3, 150), (0, 11)):
        w = torch.zeros(41, 1043 + pad, device=DEV)[:, :1043]
        w.copy_(w0)
        params, grads = [w], [g]
        for k in range(others):
            params.append(torch.randn(k % 5 + 1, 37 * k + 1, device=DEV, generator=gen))
            grads.append(torch.randn(k % 5 + 1, 37 * k + 1, device=DEV, generator=gen))
        at = others // 2
        params[0], params[at], grads[0], grads[at] = params[at], params[0], grads[at], grads[0]
        lst = training.AdamWList(params, grads, state=state, seeds=[77 if i == at else i for i in range(others + 1)])
        for _ in range(3):
            lst.fira_adamw_step(1e-3, **HYPER)
        results.append([w.contiguous(), lst.m[at], lst.v[at]] + ([] if state is F32 else [lst.m_scale[at], lst.v_scale[at]]))
    assert all(same(r, results[0]) for r in results[1:])


@pytest.mark.parametrize("state", [F32, E4M3])
def test_mixed_types_in_one_list(state):
    gen = generator(7)
    params, grads, decays = [], [], []
    for k, (a, b) in enumerate(TYPES * 3):
        params.append(matrix((k + 1, 100 + k), k % 3, a, gen, 0.02)[1])
        grads.append(matrix((k + 1, 100 + k), 0, b, gen, 1e-3)[1])
        decays.append(0.01 * k)
    states = [F32 if k % 3 == 0 else state for k in range(len(params))]
    lst = training.AdamWList(params, grads, weight_decay=decays, state=states)
    for _ in range(2):
        before = Snapshot(lst, params, grads)
        lst.fira_adamw_step(5e-3, **HYPER)
        check(lst, params, before, decays, 5e-3)


def test_empty_tensors_and_lists():
    lst = training.AdamWList([], [], device=DEV)
    lst.fira_adamw_step(1e-3)
    assert lst.t.tolist() == [1, 0]
    some = torch.ones(3, device=DEV)
    lst = training.AdamWList([torch.empty(0, 5, device=DEV), some, torch.empty(4, 0, device=DEV)], [torch.empty(0, 5, device=DEV), torch.ones(3, device=DEV), torch.empty(4, 0, device=DEV)],
                             state=[E4M3, F32, F32])
    lst.fira_adamw_step(1e-3)
    # the first step is lr in size: (g / 1) / (|g| + eps)
    assert lst.t.tolist() == [1, 0] and np.all(np.abs(f64(some) - 0.999) <= 8 * U)


@pytest.mark.parametrize("state", [F32, E4M3])
def test_zero_gradients_and_states(state):
    """0 / (0 + eps): only the decay moves the weights; a state of zeros stays one."""
    w = torch.randn(3, 500, device=DEV, generator=generator(8))
    old = w.clone()
    lst = training.AdamWList([w], [torch.zeros(3, 500, device=DEV)], weight_decay=0.5, state=state)
    lst.fira_adamw_step(0.1)
    assert torch.equal(w, old * float(np.float32(1 - 0.05))) and not lst.m[0].float().any() and not lst.v[0].float().any()
    assert state is F32 or not (lst.m_scale[0].any() or lst.v_scale[0].any())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("state", [F32, E4M3])
def test_what_is_not_finite_stays_where_it_is(state, bad):
    """The weight and state of that value are lost, all others are what they are with a zero there (the block's scale is its finite values')."""
    gen = generator(9)
    w0, g0 = 0.02 * torch.randn(4, 700, device=DEV, generator=gen), 1e-3 * torch.randn(4, 700, device=DEV, generator=gen)
    runs = []
    for x in (bad, 0.0):
        w, g = w0.clone(), g0.clone()
        g[1, 333] = g[3, 699] = x
        lst = training.AdamWList([w], [g], state=state)
        for _ in range(2):
            lst.fira_adamw_step(1e-3, **HYPER)
        runs.append((w, [lst.m[0].float(), lst.v[0].float()], [] if state is F32 else [lst.m_scale[0], lst.v_scale[0]]))
    lost = torch.zeros(4, 700, dtype=torch.bool, device=DEV)
    lost[1, 333] = lost[3, 699] = True
    assert torch.isnan(runs[0][0][lost]).all() and torch.equal(runs[0][0][~lost], runs[1][0][~lost])
    for a, b in zip(runs[0][1], runs[1][1]):
        a, b = a.view(4, 700), b.view(4, 700)
        assert not torch.isfinite(a[lost]).any() and torch.equal(a[~lost], b[~lost])
    assert same(runs[0][2], runs[1][2])


def test_small_and_large_gradients():
    """Blocks between 2^-130 and 2^60 in size, and a block of values 2^40 apart: a root above zero is never held as zero."""
    gen = generator(10)
    g = torch.randn(12, 256, device=DEV, generator=gen)
    g *= torch.tensor([2.0 ** e for e in (-120, -110, -99, -95, -60, -30, -10, 0, 20, 50, 60, 0)], device=DEV)[:, None]
    g[11] *= torch.exp2(torch.linspace(-40, 0, 256, device=DEV))
    w = torch.zeros(12, 256, device=DEV)
    lst = training.AdamWList([w], [g], state=E4M3)
    for _ in range(3):
        before = Snapshot(lst, [w], [g])
        lst.fira_adamw_step(1e-3, **HYPER)
        assert torch.isfinite(w).all()
    held = ref.e4m3(lst.v[0]).reshape(12, 256)
    assert np.all(held[4:] > 0) and not held[0].any()
    # no step is far longer than lr where m and the root are of one size, as here
    assert float(w.abs().max()) < 3 * 1e-3 * 4


def test_the_rounding_keeps_the_mean():
    """Codes of 2^18 values over 8 seeds: the mean of (held - value) / step is zero within five deviations of so many numbers in [-1, 1] with variance <= 1/4."""
    n = 1 << 18
    g = torch.empty(n, device=DEV).uniform_(0.1, 1.0, generator=generator(11))
    total = count = 0.0
    for seed in range(8):
        lst = training.AdamWList([torch.zeros(n, device=DEV)], [g.clone()], state=E4M3, seeds=[seed])
        lst.fira_adamw_step(1e-3, beta1=0.0, beta2=0.0)
        for codes in (lst.m[0], lst.v[0]):
            most, _ = ref.block_most(f64(g))
            y = f64(g) * 448.0 / most
            step = 2.0 ** (np.floor(np.log2(y)) - 3.0)
            total += float(((ref.e4m3(codes) - y) / step).sum())
            count += n
    assert abs(total / count) < 5 * 0.5 / math.sqrt(count)


def test_in_a_graph(no_automatic_collection):
    """A captured step counts on, reads the learning rate and the norm again, and is the eager step at every replay, with other work in between."""
    for state in (F32, E4M3):
        shapes = [((33, 70), 0), ((1, 511), 0), ((5, 1000), 3)]
        _, params, _, gs, _, lst, gen = problem(BF16, F32, state, 12, shapes)
        _, eager, _, egs, _, elst, _ = problem(BF16, F32, state, 12, shapes)
        clip, eclip = training.GradientList(gs), training.GradientList(egs)
        lr = torch.tensor(1e-2, device=DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norm = clip.fira_gradient_norm()
            lst.fira_adamw_step(lr, **HYPER, norm=norm, max_norm=0.05)
        for k in range(5):
            lr.fill_(1e-2 / (k + 1))
            for a, b in zip(gs, egs):
                a.copy_(torch.randn(a.shape, device=DEV, generator=gen))
                b.copy_(a)
            graph.replay()
            elst.fira_adamw_step(lr, **HYPER, norm=eclip.fira_gradient_norm(), max_norm=0.05)
            torch.cuda.synchronize()
            assert lst.t.tolist() == [k + 1, 0]
            assert same([p.contiguous() for p in params] + lst.m + lst.v, [p.contiguous() for p in eager] + elst.m + elst.v)
        del graph


def test_two_lists_on_two_streams():
    lists = []
    for seed in (13, 14):
        _, params, _, gs, _, lst, _ = problem(F32, F32, E4M3, seed)
        lists.append((params, lst))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for (_, lst), q in zip(lists, streams):
            lst.fira_adamw_step(1e-3, **HYPER, stream=q)
    torch.cuda.synchronize()
    for seed, (params, lst) in zip((13, 14), lists):
        _, want, _, _, _, alone, _ = problem(F32, F32, E4M3, seed)
        for _ in range(5):
            alone.fira_adamw_step(1e-3, **HYPER)
        assert same([p.contiguous() for p in params] + lst.m, [p.contiguous() for p in want] + alone.m) and lst.t.tolist() == [5, 0]


@pytest.mark.parametrize("state", [F32, E4M3])
def test_a_list_dropped_while_its_step_waits(state):
    """States that only the list holds, a step on a stream that is busy, and the list dropped: memory that the first stream hands out next is not the step's."""
    gen = generator(16)
    w, g = 0.02 * torch.randn(300, 1000, device=DEV, generator=gen), 1e-3 * torch.randn(300, 1000, device=DEV, generator=gen)
    want = w.clone()
    training.AdamWList([want], [g], state=state).fira_adamw_step(1e-3, **HYPER)
    side = torch.cuda.Stream()
    lst = training.AdamWList([w], [g], state=state)
    sizes = [x.numel() * x.element_size() for x in (*lst.m, *lst.v, *lst.m_scale, *lst.v_scale, lst.t) if x is not None]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    lst.fira_adamw_step(1e-3, **HYPER, stream=side)
    del lst
    others = [torch.full((n,), 77, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(8)]
    torch.cuda.synchronize()
    assert all(bool((x == 77).all()) for x in others) and torch.equal(w, want)


def test_a_run_goes_on_from_its_states():
    """Saved and put into a new list, the states go on as if nothing had happened."""
    _, params, _, gs, _, lst, _ = problem(BF16, BF16, E4M3, 15)
    for _ in range(2):
        lst.fira_adamw_step(1e-3, **HYPER)
    copy = lambda x: [None if t is None else t.clone() for t in x]  # noqa: E731
    saved = copy(params), copy(gs), copy(lst.m), copy(lst.v), copy(lst.m_scale), copy(lst.v_scale), lst.t.clone()
    lst.fira_adamw_step(1e-3, **HYPER)
    decays = [0.1 * (i % 3) for i in range(len(params))]
    again = training.AdamWList(saved[0], saved[1], weight_decay=decays, m=saved[2], v=saved[3], m_scale=saved[4], v_scale=saved[5], t=saved[6])
    again.fira_adamw_step(1e-3, **HYPER)
    assert same(copy(params) + lst.m + lst.v + lst.m_scale, saved[0] + again.m + again.v + again.m_scale)


def test_beyond_32_bit_offsets():
    """2.2e9 values, states in 8 bits: the last ones are what they are in a tensor of their own, at their place's rounding."""
    rows, cols = 66000, 33333
    n = rows * cols
    w, g = (torch.zeros(rows, cols, dtype=BF16, device=DEV) for _ in range(2))
    gen = generator(16)
    last = 4000
    w.view(-1)[-last:] = (0.02 * torch.randn(last, device=DEV, generator=gen)).to(BF16)
    g.view(-1)[-last:] = (1e-3 * torch.randn(last, device=DEV, generator=gen)).to(BF16)
    w0, g0 = f64(w.view(-1)[-last:]), f64(g.view(-1)[-last:])
    lst = training.AdamWList([w], [g], state=E4M3)
    lst.fira_adamw_step(1e-2, **HYPER)
    want = ref.adamw(w0, g0, np.zeros(last), np.zeros(last), 0, 0.0, 1e-2, 0.9, 0.999, 1e-8)
    x, off = want["w"]
    within(w.view(-1)[-last:], x, off + HALF_ULP[BF16] * (np.abs(x) + off) * (1 + 1e-3) + TINY)
    assert not w[0].any() and not w[rows // 2].any() and not lst.m[0][:100000].float().any()
    random = ref.rounding(last, 0, 1, first=n - last)[0]
    place = (n - last + np.arange(last)) // 256
    full = np.zeros((place[-1] - place[0] + 1) * 256)
    full[(n - last) % 256:(n - last) % 256 + last] = want["m"][0]
    most = np.repeat(np.abs(full.reshape(-1, 256)).max(1), 256)[(n - last) % 256:][:last]
    got = np.abs(ref.e4m3(lst.m[0][-last:]))
    assert np.mean((got >= ref.held(want["m"][0], most, random, False, -32 * U)) & (got <= ref.held(want["m"][0], most, random, False, 32 * U))) > 0.999


def test_lists_that_are_refused():
    w, g = torch.zeros(4, 300, device=DEV), torch.zeros(4, 300, device=DEV)
    f, c = torch.zeros(1200, device=DEV), torch.zeros(1200, dtype=torch.uint8, device=DEV).view(E4M3)
    scale = torch.zeros(5, device=DEV)
    held = dict(m=[c], v=[c.clone()], m_scale=[scale], v_scale=[scale.clone()])
    training.AdamWList([w], [g], **held)
    bad = [([w, w], [g, g], {}), ([w], [g[:, :299]], {}), ([w], [g.half()], {}), ([w.t()], [g.t()], {}), ([w], [g], dict(m=[f[:-1]], v=[f])), ([w], [g], dict(m=[f], v=[c])), ([w], [g], dict(m=[f], v=[f.cpu()])),
           ([w], [g], dict(m=[c], v=[c.clone()])), ([w], [g], dict(held, m_scale=[scale[:4]])), ([w], [g], dict(t=torch.zeros(1, dtype=torch.int64, device=DEV))), ([w], [g], dict(weight_decay=-1.0)),
           ([w, g], [g.clone(), w.clone()], dict(m=[f, f], v=[f.clone(), f.clone()])), ([w], [g], dict(seeds=[1, 2])), ([w], [w], {})]
    for params, grads, kw in bad:
        with pytest.raises(fira.FiraError):
            training.AdamWList(params, grads, **kw).fira_adamw_step(1e-3)
    lst = training.AdamWList([w], [g])
    for args, kw in (((math.nan,), {}), ((1e-3, 1.0), {}), ((1e-3, 0.9, 1.5), {}), ((1e-3, 0.9, 0.99, 0.0), {}), ((torch.zeros(2, device=DEV),), {}), ((torch.tensor(1e-3),), {}),
                     ((1e-3,), dict(norm=torch.tensor(1.0, device=DEV, dtype=BF16))), ((1e-3,), dict(norm=torch.tensor(1.0, device=DEV), max_norm=-1.0))):
        with pytest.raises(fira.FiraError):
            lst.fira_adamw_step(*args, **kw)
    assert lst.t.tolist() == [0, 0] and not w.any()
