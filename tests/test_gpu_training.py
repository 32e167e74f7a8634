"""The operators around the step against their definitions in 64 bits (tests/training_reference.py), where they can go wrong: one token and one
row, widths that are no multiple of a vector, leading dimensions beyond the width with NaN in between, ids outside the table,
one id for all tokens, results that are added to, values beyond fp32's squares, offsets beyond 32 bits, other streams and graphs."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01623_amd import fira, training

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)]


def matrix(rows, cols, pad, dtype, gen, scale=1.0):
    """Random values, NaN between the rows."""
    buf = torch.full((rows, cols + pad), math.nan, dtype=dtype, device=DEV)
    buf[:, :cols] = (scale * torch.randn(rows, cols, device=DEV, generator=gen)).to(dtype)
    return buf, buf[:, :cols]


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def untouched(buf, cols):
    return bool(torch.isnan(buf[:, cols:].float()).all())


def same(a, b):
    return torch.equal(a.view(torch.int16 if a.dtype == BF16 else torch.int32), b.view(torch.int16 if b.dtype == BF16 else torch.int32))


# ---- embedding -----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,rows_dtype", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim,pad", [(1, 1, 1, 0), (1, 50, 8, 0), (3, 7, 9, 3), (130, 33, 64, 0), (77, 1000, 513, 1), (600, 100, 512, 8), (65, 40, 1031, 5),
                                                  (9, 20, 5461, 0)])
def test_lookup(tokens, vocab, dim, pad, dtype, rows_dtype):
    gen = generator(tokens + dim)
    _, table = matrix(vocab, dim, pad, dtype, gen)
    buf, out = matrix(tokens, dim, pad, rows_dtype, gen)
    for ids_type in (torch.int64, torch.int32):
        ids = torch.randint(-2, vocab + 2, (tokens,), device=DEV, generator=gen).to(ids_type)
        got = training.fira_embed_lookup(table, ids, scale=0.3, out=out)
        keep = ((ids >= 0) & (ids < vocab))[:, None]
        want = torch.where(keep, table[ids.clamp(0, vocab - 1).long()].float() * float(np.float32(0.3)), torch.zeros((), device=DEV)).to(rows_dtype)
        assert got is out and torch.equal(got, want) and (pad == 0 or untouched(buf, dim))


def _skewed(tokens, vocab, gen):
    """About a third of the tokens are one id, the others uniform, some outside the table."""
    ids = torch.randint(-1, vocab + 1, (tokens,), device=DEV, generator=gen)
    ids[torch.rand(tokens, device=DEV, generator=gen) < 0.33] = vocab // 2
    return ids


@pytest.mark.parametrize("dtype,rows_dtype", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim,pad", [(1, 1, 1, 0), (1, 300, 16, 0), (5, 3, 9, 3), (64, 2, 40, 0), (65, 1, 64, 8), (700, 33, 130, 1), (1023, 260, 72, 0), (1500, 5000, 24, 0),
                                                  (2048, 257, 512, 0), (3000, 70000, 17, 0), (4999, 64, 520, 3), (9000, 1000, 33, 0), (300, 40, 1031, 5)])
def test_embed_gradient(tokens, vocab, dim, pad, dtype, rows_dtype):
    gen = generator(tokens + dim)
    _, dout = matrix(tokens, dim, pad, rows_dtype, gen)
    buf, out = matrix(vocab, dim, pad, dtype, gen)
    for ids_type, accumulate in ((torch.int64, False), (torch.int32, True)):
        ids = _skewed(tokens, vocab, gen).to(ids_type)
        old = out.clone()
        got = training.fira_embed_gradient(dout, ids, vocab, scale=1.7, out=out, accumulate=accumulate)
        want, bound = ref.embed_gradient(dout, ids, vocab, 1.7, old if accumulate else None, dtype)
        ref.within(got, want, bound)
        assert got is out and (pad == 0 or untouched(buf, dim))
        if accumulate:
            missing = torch.ones(vocab, dtype=torch.bool, device=DEV)
            missing[ids[(ids >= 0) & (ids < vocab)].long()] = False
            assert torch.equal(got[missing], old[missing])


@pytest.mark.parametrize("tokens,vocab,dim", [(300001, 1000, 8), (20000, 300000, 8), (5000, 1 << 21, 3), (70000, 50257, 20), (40000, 7, 64)])
def test_embed_gradient_of_many(tokens, vocab, dim):
    """More tokens than 256 chunks of the smallest size, more rows of a bucket than it has counters for all its wavefronts, the largest table."""
    gen = generator(tokens)
    _, dout = matrix(tokens, dim, 0, BF16, gen)
    ids = _skewed(tokens, vocab, gen)
    got = training.fira_embed_gradient(dout, ids, vocab, dtype=F32)
    want, bound = ref.embed_gradient(dout, ids, vocab, 1.0, None, F32)
    ref.within(got, want, bound)


@pytest.mark.parametrize("fill", [0, 499, -1, 500, 1 << 40, -(1 << 62)])
def test_embed_gradient_of_one_id(fill):
    """All tokens the same row, or all of them padding; an id that is a row only in its low 32 bits is outside too."""
    gen = generator(1)
    _, dout = matrix(6000, 72, 0, BF16, gen)
    ids = torch.full((6000,), fill, dtype=torch.int64, device=DEV)
    got = training.fira_embed_gradient(dout, ids, 500, dtype=F32)
    want, bound = ref.embed_gradient(dout, ids, 500, 1.0, None, F32)
    ref.within(got, want, bound)
    assert int((got != 0).any(1).sum()) == (1 if 0 <= fill < 500 else 0)
    rows = training.fira_embed_lookup(got, ids)
    assert torch.equal(rows, got[fill].expand(6000, 72) if 0 <= fill < 500 else torch.zeros(6000, 72, device=DEV))


def test_embed_gradient_of_a_row_depends_on_its_own_tokens_only():
    gen = generator(2)
    _, dout = matrix(5000, 256, 0, BF16, gen)
    ids = _skewed(5000, 900, gen)
    alone = torch.where((ids == 450) | (ids == 3), ids, torch.full_like(ids, -1))
    a, b = (training.fira_embed_gradient(dout, i, 900, dtype=F32) for i in (ids, alone))
    assert same(a[450], b[450]) and same(a[3], b[3])
    assert same(a, training.fira_embed_gradient(dout, ids, 900, dtype=F32))
    keep = ids == 450                                     # nor on where they stand among others
    assert same(a[450], training.fira_embed_gradient(dout[keep].contiguous(), ids[keep], 900, dtype=F32)[450])


@pytest.mark.parametrize("dim", [5, 64, 520])
@pytest.mark.parametrize("own", [1, 32, 33, 100, 257, 480, 512])
def test_embed_gradient_of_a_row_does_not_depend_on_the_number_of_tokens(own, dim):
    """The row of `own` tokens among no others, among a few, and among so many that the tokens are sorted; in fp32 and added to."""
    gen = generator(own)
    _, dout = matrix(3000, dim, 0, F32, gen)
    got = []
    for others in (0, 5, 513 - own if own < 512 else 1, 3000 - own):
        at = torch.randperm(own + others, device=DEV, generator=gen)[:own].sort().values
        ids = torch.randint(8, 50, (own + others,), device=DEV, generator=gen)
        ids[at] = 7
        rows = torch.randn(own + others, dim, device=DEV, generator=gen)
        rows[at] = dout[:own]
        out = torch.ones(50, dim, device=DEV)
        got.append(training.fira_embed_gradient(rows, ids, 50, scale=0.7, out=out, accumulate=True)[7].clone())
        got.append(training.fira_embed_gradient(rows, ids, 50, scale=0.7)[7])
    assert all(same(a, got[0]) for a in got[2::2]) and all(same(a, got[1]) for a in got[3::2])


def test_no_tokens():
    table = torch.randn(20, 24, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert training.fira_embed_lookup(table, none).shape == (0, 24)
    assert not training.fira_embed_gradient(torch.empty(0, 24, device=DEV), none, 20).any()
    old = table.clone()
    training.fira_embed_gradient(torch.empty(0, 24, device=DEV), none, 20, out=table, accumulate=True)
    assert torch.equal(table, old)


def test_embed_gradient_is_the_lookups():
    """<dout, lookup(E)> is linear in E, so its difference along any direction is the gradient's product with it."""
    gen = generator(3)
    table, v = torch.randn(300, 96, device=DEV, generator=gen), torch.randn(300, 96, device=DEV, generator=gen)
    ids, dout = _skewed(2000, 300, gen), torch.randn(2000, 96, device=DEV, generator=gen)
    grad = training.fira_embed_gradient(dout, ids, 300, scale=2.5)
    values = [float((training.fira_embed_lookup(table + s * v, ids, scale=2.5).double() * dout.double()).sum()) for s in (0.5, -0.5)]
    along = float((grad.double() * v.double()).sum())
    size = float((grad.double() * v.double()).square().sum().sqrt())
    assert abs(values[0] - values[1] - along) <= 1e-4 * size


def test_embedding_beyond_32_bit_offsets():
    vocab, dim = 70001, 32000                            # 2.24e9 elements
    table = torch.empty(vocab, dim, dtype=BF16, device=DEV)
    table[-3:].normal_(generator=generator(4))
    ids = torch.tensor([vocab - 1, vocab - 3, vocab, vocab - 1], device=DEV)
    rows = training.fira_embed_lookup(table, ids)
    assert torch.equal(rows[0], table[-1]) and torch.equal(rows[1], table[-3]) and not rows[2].any()
    training.fira_embed_gradient(rows, ids, vocab, out=table)
    assert torch.equal(table[-1], (rows[0].float() + rows[3].float()).to(BF16)) and torch.equal(table[-3], rows[1])
    assert not table[-2].any() and not table[vocab // 2].any() and not table[:100].any() and not table[-2000:-3].any()


# ---- norms ---------------------------------------------------------------------------------------------------------


NORM_SHAPES = [(1, 1, 0), (3, 2, 1), (2, 7, 0), (5, 64, 0), (17, 72, 8), (9, 100, 3), (200, 128, 0), (33, 250, 0), (70, 512, 0), (1000, 513, 1), (64, 1024, 8), (19, 2049, 0),
               (300, 2048, 0), (7, 4100, 3), (6, 8192, 0), (5, 11008, 0), (3, 33000, 1), (2, 70001, 0)]


@pytest.mark.parametrize("dtype,pdtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad", NORM_SHAPES)
def test_norms(rows, dim, pad, dtype, pdtype):
    gen = generator(rows + dim)
    _, x = matrix(rows, dim, pad, dtype, gen, 2.0)
    x.add_(1.0)
    buf, out = matrix(rows, dim, pad, dtype, gen)
    _, dy = matrix(rows, dim, pad, dtype, gen)
    dbuf, dx = matrix(rows, dim, pad, dtype, gen)
    w, b = ((k + 0.2 * torch.randn(dim, device=DEV, generator=gen)).to(pdtype) for k in (1.0, 0.0))
    for rms, weight, bias in ((False, w, b), (True, w, None), (False, None, None), (True, None, b)):
        y, mean, rstd = training.fira_layer_norm(x, weight, bias, eps=1e-5, rms=rms, out=out)
        r = ref.layer_norm(x, weight, bias, 1e-5, rms)
        ref.within(y, r[0], r[1])
        ref.within(rstd, r[4], r[5])
        assert (mean is None) == rms
        if not rms:
            ref.within(mean, r[2], r[3])
        accumulate = bias is None
        old = [torch.randn(dim, device=DEV, generator=gen).to(pdtype) for _ in range(2)]
        got = training.fira_layer_norm_gradient(dy, x, weight, mean, rstd, rms=rms, param_dtype=pdtype, dx=dx, dweight=old[0].clone(), dbias=old[1].clone(),
                                                accumulate=accumulate)
        r = ref.layer_norm_gradient(dy, x, weight, mean, rstd, rms, *(old if accumulate else (None, None)), pdtype)
        for k in range(3):
            ref.within(got[k], r[2 * k], r[2 * k + 1])
        assert pad == 0 or (untouched(buf, dim) and untouched(dbuf, dim))


@pytest.mark.parametrize("rows,dim", [(5000, 256), (20000, 72), (4097, 1024), (2050, 2048)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_gradients_over_many_rows(rows, dim, dtype):
    """The rows are summed in parts; each part alone, and where the last one is short."""
    gen = generator(rows)
    _, x = matrix(rows, dim, 0, dtype, gen)
    _, dy = matrix(rows, dim, 0, dtype, gen)
    w = torch.rand(dim, device=DEV, generator=gen) + 0.5
    y, mean, rstd = training.fira_layer_norm(x, w, w)
    got = training.fira_layer_norm_gradient(dy, x, w, mean, rstd)
    r = ref.layer_norm_gradient(dy, x, w, mean, rstd, False, None, None, F32)
    for k in range(3):
        ref.within(got[k], r[2 * k], r[2 * k + 1])
    again = training.fira_layer_norm_gradient(dy, x, w, mean, rstd)
    assert all(same(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("rms", [False, True])
def test_a_row_does_not_depend_on_the_others(rms):
    gen = generator(5)
    _, x = matrix(3000, 640, 0, BF16, gen)
    _, dy = matrix(3000, 640, 0, BF16, gen)
    w = torch.rand(640, device=DEV, generator=gen)
    whole = training.fira_layer_norm(x, w, rms=rms)
    part = training.fira_layer_norm(x[1234:1237], w, rms=rms)
    grads = training.fira_layer_norm_gradient(dy, x, w, whole[1], whole[2], rms=rms)
    some = training.fira_layer_norm_gradient(dy[1234:1237], x[1234:1237], w, part[1], part[2], rms=rms)
    assert same(whole[0][1234:1237], part[0]) and same(whole[2][1234:1237], part[2]) and same(grads[0][1234:1237], some[0])


@pytest.mark.parametrize("dim", [40, 513, 3000])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_a_non_finite_row_stays_alone(dim, value):
    gen = generator(6)
    _, x = matrix(9, dim, 0, F32, gen)
    _, dy = matrix(9, dim, 0, F32, gen)
    w = torch.rand(dim, device=DEV, generator=gen)
    y0, mean, rstd = training.fira_layer_norm(x, w)
    g0 = training.fira_layer_norm_gradient(dy, x, w, mean, rstd)
    x[4, dim // 2] = value
    y, mean, rstd = training.fira_layer_norm(x, w)
    g = training.fira_layer_norm_gradient(dy, x, w, mean, rstd)
    others = [0, 1, 2, 3, 5, 6, 7, 8]
    assert same(y[others], y0[others]) and same(g[0][others], g0[0][others])
    assert torch.isnan(y[4]).any() and torch.isnan(g[0][4]).any() and torch.isnan(g[1]).any()


def test_a_row_without_spread():
    """Equal values: the mean is taken off exactly, rstd is eps^-1/2; and a large mean costs the deviation nothing."""
    x = torch.full((3, 1000), 3.0, device=DEV)
    y, mean, rstd = training.fira_layer_norm(x, eps=1e-5)
    assert not y.any() and bool((mean == 3.0).all()) and torch.allclose(rstd, torch.full((3,), 1e-5, device=DEV).rsqrt(), rtol=1e-6)
    x = 1e4 + torch.randn(4, 512, device=DEV, generator=generator(7))
    _, _, rstd = training.fira_layer_norm(x, eps=0.0)
    want = 1.0 / x.double().var(1, correction=0).sqrt()
    assert float((rstd.double() / want - 1.0).abs().max()) < 1e-4        # E x^2 - mean^2 in fp32 would be off by several


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradients_are_the_norms(rms):
    """Central differences of <dy, y> along random directions: step 1e-2, so that the curvature counts 1e-4 and the rounding of y / step 1e-5."""
    gen = generator(8)
    x, dy, vx = (torch.randn(40, 320, device=DEV, generator=gen) for _ in range(3))
    w, b, vw, vb = (torch.randn(320, device=DEV, generator=gen) for _ in range(4))
    _, mean, rstd = training.fira_layer_norm(x, w, b, rms=rms)
    dx, dw, db = training.fira_layer_norm_gradient(dy, x, w, mean, rstd, rms=rms)
    h = 1e-2

    def loss(s, which):
        args = [x + s * vx if which == 0 else x, w + s * vw if which == 1 else w, b + s * vb if which == 2 else b]
        return float((training.fira_layer_norm(*args, rms=rms)[0].double() * dy.double()).sum())

    for which, (g, v) in enumerate(((dx, vx), (dw, vw), (db, vb))):
        terms = g.double() * v.double()
        assert abs((loss(h, which) - loss(-h, which)) / (2 * h) - float(terms.sum())) <= 1e-3 * float(terms.square().sum().sqrt())


def test_norms_of_nothing():
    w = torch.ones(24, device=DEV)
    y, mean, rstd = training.fira_layer_norm(torch.empty(0, 24, device=DEV), w)
    assert y.shape == (0, 24) and mean.shape == (0,)
    dx, dw, db = training.fira_layer_norm_gradient(y, y, w, mean, rstd)
    assert dx.shape == (0, 24) and not dw.any() and not db.any()
    old = torch.randn(24, device=DEV)
    _, dw, db = training.fira_layer_norm_gradient(y, y, w, mean, rstd, dweight=old.clone(), dbias=old.clone(), accumulate=True)
    assert torch.equal(dw, old) and torch.equal(db, old)


def test_norms_beyond_32_bit_offsets():
    ld, dim = (1 << 30) + 7, 1000
    buf = torch.empty(3 * ld, dtype=BF16, device=DEV)
    x = buf.as_strided((3, dim), (ld, 1))
    x.normal_(generator=generator(9))
    y, mean, rstd = training.fira_layer_norm(x)
    dense = training.fira_layer_norm(x.contiguous())
    assert same(y, dense[0]) and same(mean, dense[1]) and same(rstd, dense[2])
    a = training.fira_layer_norm_gradient(x, x, None, mean, rstd)
    b = training.fira_layer_norm_gradient(x.contiguous(), x.contiguous(), None, mean, rstd)
    assert all(same(p, q) for p, q in zip(a, b))


# ---- gradient norm and clipping ------------------------------------------------------------------------------------


def _gradients(shapes, dtypes, pad, gen, scale=1.0):
    made = [matrix(m, n, pad, t, gen, scale) for (m, n), t in zip(shapes, dtypes)]
    return [m[0] for m in made], [m[1] for m in made]


def _norm64(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


LISTS = [[(1, 1)], [(3, 5), (1, 7)], [(1, 100), (64, 64), (33, 9), (2, 4100)], [(300, 517), (1, 300), (517, 300), (700, 8)], [(5, 3)] * 230 + [(1024, 1376)]]


@pytest.mark.parametrize("shapes", LISTS)
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_clip(shapes, pad):
    gen = generator(len(shapes) + pad)
    types = [(F32, BF16)[i % 2] for i in range(len(shapes))]
    bufs, grads = _gradients(shapes, types, pad, gen)
    norm = _norm64(grads)
    lst = training.GradientList(grads)
    assert abs(float(lst.fira_gradient_norm()) / norm - 1.0) <= 4 * ref.U
    before = [g.clone() for g in grads]
    assert abs(float(lst.fira_clip_gradients(norm * 1.001)) / norm - 1.0) <= 4 * ref.U
    assert all(same(a, b.contiguous()) for a, b in zip(before, [g.contiguous() for g in grads]))
    # elsewhere, in every type
    for out_types in ((F32, F32), (BF16, BF16), (BF16, F32)):
        obufs, outs = _gradients(shapes, [out_types[i % 2] for i in range(len(shapes))], 5, gen)
        other = training.GradientList(grads, outs)
        for limit in (norm / 3.0, norm * 2.0, math.inf):
            got = float(other.fira_clip_gradients(limit))
            assert abs(got / norm - 1.0) <= 4 * ref.U
            for g, o in zip(grads, outs):
                want = ref.f64(g) * min(1.0, limit / norm)
                ref.within(o, want, (4 * ref.U + ref.HALF_ULP[o.dtype]) * np.abs(want) + ref.TINY)
        assert all(untouched(b, o.shape[1]) for b, o in zip(obufs, outs))
    got = float(lst.fira_clip_gradients(norm / 7.0))
    assert abs(got / norm - 1.0) <= 4 * ref.U
    for g, b in zip(grads, before):
        want = ref.f64(b) / 7.0
        ref.within(g, want, (5 * ref.U + ref.HALF_ULP[g.dtype]) * np.abs(want) + ref.TINY)
    assert pad == 0 or all(untouched(b, g.shape[1]) for b, g in zip(bufs, grads))


@pytest.mark.parametrize("scale", [1e-30, 1e25])
def test_squares_leave_the_range_of_fp32(scale):
    grads = [torch.randn(100, 77, device=DEV, generator=generator(10)) * scale, torch.randn(33, device=DEV).to(BF16) * scale]
    norm = _norm64(grads)
    before = grads[0].clone()
    assert abs(float(training.GradientList(grads).fira_clip_gradients(norm / 2)) / norm - 1.0) <= 4 * ref.U
    assert torch.allclose(grads[0], before * 0.5, rtol=1e-6, atol=0.0)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite(value):
    g = torch.randn(40, 50, device=DEV)
    g[3, 4] = value
    before, out = g.clone(), torch.empty(40, 50, dtype=BF16, device=DEV)
    for lst in (training.GradientList([g]), training.GradientList([g], [out])):
        got = float(lst.fira_clip_gradients(1.0))
        assert math.isnan(got) if math.isnan(value) else got == math.inf
    assert same(g, before) and same(out, before.to(BF16))


def test_lists_of_nothing():
    assert float(training.GradientList([], device=DEV).fira_gradient_norm()) == 0.0
    empty = [torch.empty(0, 5, device=DEV), torch.empty(4, 0, dtype=BF16, device=DEV)]
    assert float(training.GradientList(empty).fira_clip_gradients(1.0)) == 0.0
    zero = torch.zeros(9, device=DEV)
    assert float(training.GradientList([zero, torch.zeros((), device=DEV)] + empty).fira_clip_gradients(0.0)) == 0.0 and not zero.any()
    g = torch.full((3,), 2.0, device=DEV)
    assert abs(float(training.GradientList([g]).fira_clip_gradients(0.0)) - math.sqrt(12.0)) < 1e-6 and not g.any()


def test_a_gradient_of_more_than_2_31_values():
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=BF16, device=DEV)
    g[[0, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1]] = 2.0
    lst = training.GradientList([g, torch.ones(5, device=DEV)])
    assert abs(float(lst.fira_clip_gradients(2.5)) - 5.0) < 1e-6
    assert float(g[0]) == float(g[1 << 30]) == float(g[1 << 31]) == float(g[n - 1]) == 1.0 and float(g.sum(dtype=torch.float64)) == 5.0


def test_clip_gives_the_same_bits_again():
    _, grads = _gradients([(1000, 1376)] * 7 + [(77, 3001)], [BF16] * 4 + [F32] * 4, 0, generator(11))
    a, b = ([g.clone() for g in grads] for _ in range(2))
    na, nb = training.GradientList(a).fira_clip_gradients(1.0), training.GradientList(b).fira_clip_gradients(1.0)
    assert same(na, nb) and all(same(p, q) for p, q in zip(a, b))


# ---- streams, graphs, strides --------------------------------------------------------------------------------------


def _everything(s, stream=None):
    rows = training.fira_embed_lookup(s["table"], s["ids"], scale=2.0, stream=stream)
    y, mean, rstd = training.fira_layer_norm(rows, s["w"], s["w"], stream=stream)
    dx, dw, db = training.fira_layer_norm_gradient(y, rows, s["w"], mean, rstd, stream=stream)
    de = training.fira_embed_gradient(dx, s["ids"], s["table"].shape[0], scale=2.0, stream=stream)
    outs = [torch.empty_like(t) for t in (de, dw, db)]
    norm = training.GradientList([de, dw, db], outs).fira_clip_gradients(0.5, stream=stream)
    return [rows, y, mean, rstd, dx, dw, db, de, norm] + outs


def _inputs(tokens=3000):
    gen = generator(12)
    return dict(table=torch.randn(700, 264, device=DEV, generator=gen).to(BF16), ids=_skewed(tokens, 700, gen), w=torch.rand(264, device=DEV, generator=gen).to(BF16))


def test_on_another_stream():
    s = _inputs()
    want = _everything(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        later = {k: torch.empty_like(v) for k, v in s.items()}
        torch.cuda._sleep(20_000_000)                    # what follows on the default stream would run before the inputs are there
        for k, v in s.items():
            later[k].copy_(v)
    got = _everything(later, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("tokens", [100, 3000])
def test_in_a_graph(tokens, no_automatic_collection):
    s = _inputs(tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _everything(s)                                   # the library and its kernels are loaded
        held = [torch.empty(t, dtype=d, device=DEV) for t, d in (((700, 264), BF16), ((264,), BF16), ((264,), BF16))]
        kept = training.GradientList(held, [torch.empty_like(t) for t in held])

        def run():
            rows = training.fira_embed_lookup(s["table"], s["ids"], scale=2.0)
            y, mean, rstd = training.fira_layer_norm(rows, s["w"], s["w"])
            dx, _, _ = training.fira_layer_norm_gradient(y, rows, s["w"], mean, rstd, dweight=held[1], dbias=held[2])
            training.fira_embed_gradient(dx, s["ids"], 700, scale=2.0, out=held[0])
            return [rows, y, dx, kept.fira_clip_gradients(0.5)] + held + kept._keep[1]

        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run()
    torch.cuda.synchronize()
    for k in range(4):
        s["ids"].copy_(_skewed(tokens, 700, generator(20 + k)))
        s["table"].mul_(1.25)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for t in held:
            t.normal_()
        with torch.cuda.stream(side):
            want = run()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(got, want)), k


def test_inputs_of_any_strides():
    """More dimensions, expanded and permuted views: as their dense copies."""
    gen = generator(13)
    x = torch.randn(6, 5, 48, device=DEV, generator=gen)
    w = torch.rand(48, device=DEV, generator=gen)
    for view in (x.transpose(0, 1), x[:, 1:4], x[::2], x[:, :, 8:40], x[0:1].expand(6, 5, 48), x[:, :, :1], x[2, 3]):
        wv = w[:view.shape[-1]]
        a, b = training.fira_layer_norm(view, wv), training.fira_layer_norm(view.contiguous(), wv)
        assert all(same(p, q) for p, q in zip(a, b)) and a[0].shape == view.shape and a[1].shape == view.shape[:-1]
        a, b = (training.fira_layer_norm_gradient(v, v, wv, a[1], a[2]) for v in (view, view.contiguous()))
        assert all(same(p, q) for p, q in zip(a, b))
    ids = torch.randint(0, 30, (8, 9), device=DEV, generator=gen)
    table = torch.randn(30, 48, device=DEV, generator=gen)
    assert torch.equal(training.fira_embed_lookup(table, ids[:, :-1]), table[ids[:, :-1]])
    assert torch.equal(training.fira_embed_lookup(table.t().contiguous().t(), ids), table[ids])
    dout = torch.ones(1, device=DEV).expand(8, 8, 48)
    got = training.fira_embed_gradient(dout, ids[:, 1:], 30)
    assert torch.equal(got, torch.bincount(ids[:, 1:].flatten(), minlength=30).float()[:, None].expand(30, 48))


def test_refusals_of_the_binding():
    x, w = torch.randn(4, 16, device=DEV), torch.ones(16, device=DEV)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    mean, rstd = torch.zeros(4, device=DEV), torch.ones(4, device=DEV)
    t = training
    bad = [
        (fira.FIRA_ERR_DTYPE, lambda: t.fira_embed_lookup(x.half(), ids)),
        (fira.FIRA_ERR_DTYPE, lambda: t.fira_embed_lookup(x, ids.to(torch.int16))),
        (fira.FIRA_ERR_DTYPE, lambda: t.fira_embed_lookup(x, ids, dtype=BF16, out=torch.empty(4, 16, device=DEV))),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_embed_lookup(x[0], ids)),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_embed_lookup(x, ids, out=torch.empty(5, 16, device=DEV))),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_embed_lookup(x, ids, out=torch.empty(16, 4, device=DEV).t())),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_embed_lookup(x, ids.cpu())),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_embed_lookup(x.cpu(), ids.cpu())),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_embed_lookup(x, ids, scale=math.inf)),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_embed_gradient(x, ids[:3], 10)),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_embed_gradient(x, ids, 0)),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_embed_gradient(x, ids, 10, accumulate=True)),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_embed_gradient(x, ids, 10, workspace=torch.empty(256, device=DEV))),
        (fira.FIRA_ERR_WORKSPACE, lambda: t.fira_embed_gradient(x, ids, 10, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_layer_norm(x, w[:8])),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_layer_norm(x[:, :0])),
        (fira.FIRA_ERR_DTYPE, lambda: t.fira_layer_norm(x, w, w.to(BF16))),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_layer_norm(x, w, eps=-1.0)),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_layer_norm_gradient(x, x, w, None, rstd)),
        (fira.FIRA_ERR_SHAPE, lambda: t.fira_layer_norm_gradient(x, x, w, mean, rstd[:3])),
        (fira.FIRA_ERR_DTYPE, lambda: t.fira_layer_norm_gradient(x.to(BF16), x, w, mean, rstd)),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.fira_layer_norm_gradient(x, x, w, mean, rstd, accumulate=True)),
        (fira.FIRA_ERR_DTYPE, lambda: t.GradientList([x.half()])),
        (fira.FIRA_ERR_SHAPE, lambda: t.GradientList([x.t()])),
        (fira.FIRA_ERR_SHAPE, lambda: t.GradientList([x], [x[:2]])),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.GradientList([x], [])),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.GradientList([])),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.GradientList([x]).fira_clip_gradients(-1.0)),
        (fira.FIRA_ERR_INVALID_ARG, lambda: t.GradientList([x]).fira_clip_gradients(math.nan)),
    ]
    for k, (status, call) in enumerate(bad):
        with pytest.raises(fira.FiraError) as ei:
            call()
        assert ei.value.status == status, (k, str(ei.value))
