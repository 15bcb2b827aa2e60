"""Layer norm of rows whose spread is small beside their mean, on the GPU."""
import math

import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers

pytestmark = pytest.mark.gpu
EPS = 1e-5
COLUMNS = [3, 7, 56, 100, 480, 921, 2050, 9000]


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


@pytest.mark.parametrize("c", COLUMNS)
@pytest.mark.parametrize("value", [1000.0, 0.1, -777.7])
def test_constant_rows(c, value):
    """The mean is off by (k + 2) u |x| before it is corrected, the correction by k + 2
    roundings of that; rstd is at most eps^-1/2."""
    x = torch.full((5, c), value).cuda()
    y, (mean, _) = layers.layer_norm(x, eps=EPS, save=True)
    k = refs.norm_depth(c)
    bound = ((k + 2) * refs.U) ** 2 * abs(value) / math.sqrt(EPS)
    print(f"largest {y.abs().max().item():.3e}, bound {bound:.3e}", flush=True)
    assert (y.abs() <= bound).all()
    assert torch.equal(mean, x[:, 0])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("c", COLUMNS)
def test_rows_of_small_spread(c, dtype):
    """Values a few steps of the type around 1000.  Their distances from the mean,
    whose error is e = (k + 2) u |mean| at first, are exact in 32 bits (both lie within a
    factor of two); the mean distance is subtracted with k + 2 roundings of the
    distances' mean, and the variance, a difference of two sums, is off by k + 4
    roundings of them."""
    gen = torch.Generator().manual_seed(c)
    step = {"f32": 2.0 ** -14, "f16": 0.5, "bf16": 4.0}[dtype]
    x = 1000.0 + step * torch.randint(-4, 5, (9, c), generator=gen).double()
    x = x.to(refs.TDT[dtype])
    y = layers.layer_norm(x.cuda(), eps=EPS)
    ref, h, mean, rstd = refs.layer_norm(x.double(), torch.ones(c).double(), torch.zeros(c).double(), EPS)
    k = refs.norm_depth(c)
    far = (x.double() - mean).abs() + (k + 2) * refs.U * mean.abs()
    moved = refs.U * ((k + 3) * far.mean(1, keepdim=True) + far)
    spread = (k + 4) * refs.U * 2 * (far ** 2).mean(1, keepdim=True) * rstd ** 2
    err = moved * rstd + (h.abs() + moved * rstd) * (spread + 8 * refs.U)
    half = refs.HALF[dtype]
    refs.within(y, ref, err + half * (ref.abs() + err) + refs.TINY[dtype], "y")


@pytest.mark.parametrize("c", [7, 480, 921, 9000])
@pytest.mark.parametrize("size", [1e18, 1e24, 1e30])
def test_rows_whose_squares_pass_the_range(c, size):
    """Where the sum of squares, about c size^2, passes 3.4e38, rstd is 0 and y is beta,
    as the definition in 32 bits gives it; below that, y is as exact as ever."""
    gen = torch.Generator().manual_seed(c)
    x, beta = torch.randn(5, c, generator=gen) * size, torch.randn(c, generator=gen)
    y = layers.layer_norm(x.cuda(), None, beta.cuda(), eps=EPS)
    if c * size ** 2 > 4e38:
        assert torch.equal(y.cpu(), beta.expand(5, c))
        return
    ref, h, mean, rstd = refs.layer_norm(x.double(), torch.ones(c).double(), beta.double(), EPS)
    he = refs.norm_h_error(x.double(), h, rstd, c)
    refs.within(y, ref, he + 4 * refs.U * (h.abs() + beta.double().abs()), "y")
