"""The norm gradients' sums over rows: with whole numbers for x, dy and the mean, and powers of two for rstd, every product and every sum is exact in
fp32 whatever the order, so that a row lost, counted twice or added to another column shows, however many rows there are."""
import pytest
import torch

from paper_2410_01623_amd import training

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# widths of every way in which a row is held, odd ones among them; rows of one launch without a workspace, and of parts of which the last is short
SHAPES = [(rows, dim) for dim in (1, 7, 9, 31, 64, 65, 100, 128, 250, 256, 257, 511, 513, 1000, 2048, 2049) for rows in (1, 33, 512, 513, 3001, 20001)]
SHAPES += [(rows, dim) for dim in (4095, 4100, 8191, 8200, 16384) for rows in (3, 511, 514, 2500)]
SHAPES += [(rows, dim) for dim in (16385, 33001) for rows in (1, 65, 700)]


@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_every_row_counts_once(rows, dim, dtype, pdtype):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows + 7 * dim)

    def whole(most, *shape):
        return torch.randint(-most, most + 1, shape, device=DEV, generator=gen)

    x, dy = whole(8, rows, dim).to(dtype), whole(4, rows, dim).to(dtype)
    mean, rstd = whole(2, rows).float(), torch.exp2(whole(1, rows).float())
    old = [whole(4, dim).to(pdtype) for _ in range(2)]
    weight = torch.ones(dim, dtype=pdtype, device=DEV)
    for rms in (False, True):
        h = (x.double() - (0.0 if rms else mean.double()[:, None])) * rstd.double()[:, None]
        want = ((dy.double() * h).sum(0), dy.double().sum(0))
        _, dw, db = training.fira_layer_norm_gradient(dy, x, weight, None if rms else mean, rstd, rms=rms)
        assert torch.equal(dw, want[0].to(pdtype)) and torch.equal(db, want[1].to(pdtype))
        _, dw, db = training.fira_layer_norm_gradient(dy, x, weight, None if rms else mean, rstd, rms=rms, dweight=old[0].clone(), dbias=old[1].clone(), accumulate=True)
        assert torch.equal(dw, (want[0] + old[0].double()).to(pdtype)) and torch.equal(db, (want[1] + old[1].double()).to(pdtype))
