"""The block norm at every number of threads and vectors that a row is held by, forward and in the gradient, and as a block without gate and post norm has it:
root-mean-square norm, a weight, gradients from both results; against the definition in 64 bits (tests/model_reference.py)."""
import pytest
import torch

from paper_2410_01623_amd import fira, training

import model_reference as ref
import test_gpu_block_norm as base
from test_gpu_block_norm import F32, NAMES, TYPES
from training_reference import within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(9, 257, 0), (5, 1025, 3), (4, 2560, 0), (5, 2561, 1), (3, 3584, 8), (4, 3585, 0), (5, 3590, 1), (3, 4095, 0), (300, 4096, 0), (4, 4097, 3), (3, 5119, 1), (5, 5120, 0), (4, 5121, 0),
          (3, 6144, 8), (5, 6145, 1), (4, 7167, 0), (3, 7168, 0), (5, 7169, 3), (4, 8191, 0), (3, 8193, 0), (4, 10241, 1), (3, 16383, 0), (2, 16385, 0)]


@pytest.mark.parametrize("dtype,pdtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad", SHAPES)
def test_forward(rows, dim, pad, dtype, pdtype):
    base.test_forward(rows, dim, pad, dtype, pdtype)


@pytest.mark.parametrize("dtype,pdtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad", SHAPES)
def test_gradient(rows, dim, pad, dtype, pdtype):
    base.test_gradient(rows, dim, pad, dtype, pdtype)


@pytest.mark.parametrize("dtype,pdtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad", [(1, 1, 0), (5, 7, 2), (1, 2048, 0), (33, 64, 0), (70, 513, 3), (600, 1024, 0), (9, 2049, 0), (40, 4096, 8), (3, 11008, 0), (2, 20000, 0)])
def test_rms_norm_alone(rows, dim, pad, dtype, pdtype):
    """r = x + block, y = weight r / |r|: the call's defaults.  The gradient reads no block."""
    gen = base.generator(rows + dim)
    (_, x), (_, block) = base.matrix(rows, dim, pad, dtype, gen), base.matrix(rows, dim, 0, dtype, gen, 0.7)
    x += 0.3
    weight = (1.0 + 0.3 * torch.randn(dim, device=DEV, generator=gen)).to(pdtype)
    v = dict(dict.fromkeys(NAMES), weight=weight)
    got = training.fira_block_norm(x, block, weight)
    for a, b in zip(got, ref.block_norm(x, block, v, "rms", "none", 1e-5, 1e-5, 1.0, 1.0)):
        assert (a is None) == (b is None)
        if a is not None:
            within(a, *b)
    r = got.residual
    (_, dr), (_, dy) = base.matrix(rows, dim, pad, dtype, gen), base.matrix(rows, dim, 0, dtype, gen)
    stats = (None, got.rstd, None, None)
    for from_stream, bias, add in ((dr, False, False), (dr, False, True), (None, False, False), (dr, True, True)):
        old = {k: torch.randn(dim, device=DEV, generator=gen).to(pdtype) for k in (("weight", "bias") if bias else ("weight",))} if add else None
        given = {f"d{k}": t.clone() for k, t in (old or {}).items()}
        back = training.fira_block_norm_gradient(from_stream, dy, r, block, weight, None, got.rstd, bias=bias, accumulate=add, **given)
        want, sums = ref.block_norm_gradient(from_stream, dy, r, block, v, stats, "rms", "none", 1.0, 1.0, old, pdtype)
        within(back.dx, *want[0])
        within(back.dblock, *want[1])
        within(back.dweight, *sums["weight"])
        assert torch.equal(back.dx, back.dblock) and [back.dgate, back.dpost_weight, back.dpost_bias] == [None] * 3
        if bias:
            within(back.dbias, *sums["bias"])
        else:
            assert back.dbias is None


@pytest.mark.parametrize("dim", [64, 2049, 9000])
def test_no_block_is_read_that_is_not_needed(dim):
    """The C entry point takes no block where neither a gate nor a post norm wants its values."""
    gen = base.generator(dim)
    rows = 37
    r, dr, dy = (torch.randn(rows, dim, device=DEV, generator=gen) for _ in range(3))
    weight, rstd = torch.randn(dim, device=DEV, generator=gen), torch.rand(rows, device=DEV, generator=gen) + 0.5
    want = training.fira_block_norm_gradient(dr, dy, r, r, weight, None, rstd)
    lib = fira.load_library()
    d = fira.fira_block_norm_desc(rows, dim, fira.FIRA_F32, fira.FIRA_F32, fira.FIRA_RMS_NORM, fira.FIRA_NO_NORM, 0.0, 0.0, 1.0, 1.0)
    dx, db, dw = torch.empty_like(r), torch.empty_like(r), torch.empty_like(weight)
    workspace = torch.empty(lib.fira_block_norm_gradient_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    vectors, to = fira.fira_block_norm_params(weight=weight.data_ptr()), fira.fira_block_norm_params(weight=dw.data_ptr())
    assert lib.fira_block_norm_gradient(d, dr.data_ptr(), dim, dy.data_ptr(), dim, r.data_ptr(), dim, None, 0, vectors, None, rstd.data_ptr(), None, None, dx.data_ptr(), dim, db.data_ptr(),
                                        dim, to, 0, workspace.data_ptr(), workspace.numel(), torch.cuda.current_stream().cuda_stream) == fira.FIRA_OK
    assert base.same((dx, db, dw), (want.dx, want.dblock, want.dweight))
