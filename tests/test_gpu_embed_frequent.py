"""The embedding gradient of rows that very many tokens name: a row of more than 8192 tokens is summed in pieces of 64 tokens, of more than 16384
in pieces of 128 and so on, at most 256 of them.  Small whole numbers have sums that fp32 holds exactly in any order, so that a token
lost or counted twice shows in every column; other values are held to the roundings of the order in which they are added."""
import numpy as np
import pytest
import torch

from paper_2410_01623_amd import training

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)]
U = 2.0 ** -24
HALF_ULP = {F32: 0.0, BF16: 2.0 ** -8}     # of the last rounding, where fp32 arithmetic does not end in one already


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def same(a, b):
    return torch.equal(a.view(torch.int16 if a.dtype == BF16 else torch.int32), b.view(torch.int16 if b.dtype == BF16 else torch.int32))


def frequent(counts, others, vocab, gen):
    """Ids of which `counts` (row: number) are named so often, `others` more of the other rows or outside the table, in random order."""
    rest = torch.randint(len(counts) - 1, vocab + 1, (others,), device=DEV, generator=gen)      # (the rows of `counts` are 0, 1, ...)
    rest[rest == len(counts) - 1] = -1
    ids = torch.cat([torch.full((n,), v, device=DEV, dtype=torch.int64) for v, n in enumerate(counts)] + [rest])
    return ids[torch.randperm(ids.numel(), device=DEV, generator=gen)]


def sums64(dout, ids, vocab):
    keep = (ids >= 0) & (ids < vocab)
    total = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=DEV)
    return total.index_add_(0, ids[keep], dout[keep].double())


def whole(rows, cols, dtype, gen, pad=0):
    buf = torch.full((rows, cols + pad), float("nan"), dtype=dtype, device=DEV)[:, :cols]
    return buf.copy_(torch.randint(-4, 5, (rows, cols), device=DEV, generator=gen))


COUNTS = [(8192,), (8193,), (16384, 8200), (16385, 8192, 33), (40000,), (10000, 20000, 9000)]


@pytest.mark.parametrize("dtype,rows_dtype", TYPES)
@pytest.mark.parametrize("dim,pad", [(24, 0), (200, 0), (264, 8), (520, 0), (1024, 0), (1031, 1)])
@pytest.mark.parametrize("counts", COUNTS)
def test_every_token_of_a_frequent_row_counts_once(counts, dim, pad, dtype, rows_dtype):
    gen = generator(sum(counts) + dim)
    vocab = 300
    ids = frequent(counts, 3001, vocab, gen)
    dout = whole(ids.numel(), dim, rows_dtype, gen, pad)
    want = sums64(dout, ids, vocab)
    got = training.fira_embed_gradient(dout, ids, vocab, scale=0.5, dtype=dtype)
    assert torch.equal(got, (0.5 * want).to(dtype))
    old = whole(vocab, dim, dtype, gen, pad)
    got = training.fira_embed_gradient(dout, ids.int(), vocab, scale=2.0, out=old.clone(), accumulate=True)
    assert torch.equal(got, (2.0 * want + old.double()).to(dtype))


@pytest.mark.parametrize("dtype,rows_dtype", TYPES)
@pytest.mark.parametrize("dim", [264, 1024])
def test_a_batch_of_one_token(dim, dtype, rows_dtype):
    gen = generator(dim)
    dout = whole(131072, dim, rows_dtype, gen)
    ids = torch.full((131072,), 17, dtype=torch.int32, device=DEV)
    want = torch.zeros(40, dim, dtype=torch.float64, device=DEV)
    want[17] = dout.double().sum(0)
    assert torch.equal(training.fira_embed_gradient(dout, ids, 40, dtype=dtype), want.to(dtype))


def additions(n):
    """Roundings that a value of a row of n tokens goes through while it is summed: those of its piece, of one of eight parts, of the join."""
    n = n.astype(np.int64)
    size = np.full_like(n, 32)
    while (n > 256 * size).any():
        size[n > 256 * size] *= 2
    pieces = -(-n // size)
    return np.where(n > 32, size - 1 + -(-pieces // 8) - 1 + 7, np.maximum(n - 1, 0))


@pytest.mark.parametrize("dtype,rows_dtype", TYPES)
@pytest.mark.parametrize("counts", [(700,), (8193, 1000, 33, 31), (70000, 9000)])
@pytest.mark.parametrize("dim", [72, 520, 1031])
def test_roundings_of_frequent_rows(dim, counts, dtype, rows_dtype):
    """One rounding an addition, one for the scale, one for what is added to, one for the result's type."""
    gen = generator(sum(counts) + dim)
    vocab = 500
    ids = frequent(counts, 2000, vocab, gen)
    dout = torch.randn(ids.numel(), dim, device=DEV, generator=gen).to(rows_dtype)
    steps = torch.from_numpy(additions(torch.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab).cpu().numpy())).to(DEV)[:, None]
    scale = float(np.float32(1.7))
    want, size = scale * sums64(dout, ids, vocab), scale * sums64(dout.abs(), ids, vocab)
    for accumulate in (False, True):
        out = torch.randn(vocab, dim, device=DEV, generator=gen).to(dtype)
        ref = want + out.double() if accumulate else want
        off = (steps + 1) * U * size + (U * ref.abs() if accumulate else 0.0)
        off = 1.001 * (off + HALF_ULP[dtype] * (ref.abs() + off)) + 1e-37
        got = training.fira_embed_gradient(dout, ids, vocab, scale=1.7, out=out, accumulate=accumulate)
        assert float(((got.double() - ref).abs() - off).max()) <= 0.0


@pytest.mark.parametrize("own", [8192, 8193, 20000])
def test_a_frequent_rows_bits_depend_on_its_own_tokens_only(own):
    """... not on how many others there are, nor on how wide the rows are and which kernel sums them."""
    gen = generator(own)
    dim = 520
    mine = torch.randn(own, dim, device=DEV, generator=gen).to(BF16)
    got = []
    for others in (0, 1, 6000):
        at = torch.randperm(own + others, device=DEV, generator=gen)[:own].sort().values
        ids = torch.randint(8, 50, (own + others,), device=DEV, generator=gen)
        ids[at] = 7
        rows = torch.randn(own + others, dim, device=DEV, generator=gen).to(BF16)
        rows[at] = mine
        got.append(training.fira_embed_gradient(rows, ids, 50, dtype=BF16)[7])
        narrow = training.fira_embed_gradient(rows[:, :200], ids, 50, dtype=BF16)[7]
        assert same(got[-1][:200], narrow)
    assert all(same(a, got[0]) for a in got[1:])
