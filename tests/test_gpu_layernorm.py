"""Layer norm on the GPU, forward and backward, against the 64-bit reference,
within bounds derived in token_refs."""
import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _rows(rows, pitch, offset, c, gen, dtype, scale=1.0, mean=0.0):
    """[rows, c] view with a pitch, `offset` elements into its storage, all around it NaN."""
    x = torch.randn(rows, c, generator=gen) * scale + mean
    flat = torch.full((offset + rows * pitch + 8,), float("nan"))
    v = flat[offset:offset + rows * pitch].view(rows, pitch)[:, :c] if rows else flat[:0].view(0, c)
    v.copy_(x)
    dev = flat.to(refs.TDT[dtype]).cuda()
    return dev, dev[offset:offset + rows * pitch].view(rows, pitch)[:, :c] if rows else dev[:0].view(0, c)


SHAPES = [
    # rows, c, pitch of x, offset of x in elements
    (1, 1, 1, 0), (3, 7, 7, 0), (5, 8, 8, 0), (98, 512, 512, 0), (33, 460, 464, 0),
    (1, 2048, 2048, 0), (17, 2050, 2056, 0), (9, 4096, 4096, 0), (4, 8192, 8192, 0),
    (3, 9000, 9000, 0), (40, 921, 921, 1), (7, 1500, 1501, 0), (2000, 64, 64, 0), (300, 100, 104, 8),
    (129, 256, 256, 3), (2, 65, 65, 0), (20000, 24, 24, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,c,pitch,offset", SHAPES)
def test_layer_norm_forward_and_backward(rows, c, pitch, offset, dtype):
    gen = torch.Generator().manual_seed(rows * 131 + c)
    _, x = _rows(rows, pitch, offset, c, gen, dtype, 2.0, 1.5)
    _, dy = _rows(rows, c, 0, c, gen, dtype)
    gamma, beta = torch.randn(c, generator=gen), torch.randn(c, generator=gen)
    y, saved = layers.layer_norm(x, gamma.cuda(), beta.cuda(), EPS, save=True)
    dx, dg, db = layers.layer_norm_backward(dy, x, gamma.cuda(), saved)
    torch.cuda.synchronize()
    x64, dy64, g64, b64 = x.double().cpu(), dy.double().cpu(), gamma.double(), beta.double()
    ref, h, mean, rstd = refs.layer_norm(x64, g64, b64, EPS)
    half, k = refs.HALF[dtype], refs.norm_depth(c)
    he = refs.norm_h_error(x64, h, rstd, c)
    bound = he * g64.abs() + 3 * refs.U * (h.abs() * g64.abs() + b64.abs())
    refs.within(y, ref, bound + half * (ref.abs() + bound) + refs.TINY[dtype], "y")
    refs.within(saved[0], mean[:, 0], (k + 2) * refs.U * x64.abs().mean(1), "mean")
    dx64, dg64, db64 = refs.layer_norm_grads(dy64, h, rstd, g64)
    w = (dy64 * g64).abs()
    mw, mwh = w.mean(1, keepdim=True), (w * h.abs()).mean(1, keepdim=True)
    err = rstd * (4 * refs.U * (w + mw + h.abs() * mwh) + (k + 4) * refs.U * (mw + h.abs() * mwh) +
                  he * mwh + h.abs() * (w * he).mean(1, keepdim=True) +
                  (he.max(1, keepdim=True).values + 8 * refs.U) * (w + mw + h.abs() * mwh))
    refs.within(dx, dx64, err + half * (dx64.abs() + err) + refs.TINY[dtype], "dx")
    deep = (rows + 64) * refs.U
    refs.within(dg, dg64, (dy64.abs() * (he + deep * h.abs())).sum(0), "dgamma")
    refs.within(db, db64, deep * dy64.abs().sum(0), "dbeta")


def test_weights_may_be_absent_and_the_result_may_replace_the_input():
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(50, 96, generator=gen).cuda()
    y = layers.layer_norm(x)
    ref = refs.layer_norm(x.double().cpu(), torch.ones(96).double(), torch.zeros(96).double(), EPS)[0]
    refs.within(y, ref, 2e-6 * (1 + ref.abs()), "plain")
    z = x.clone()
    assert layers.layer_norm(z, out=z) is z
    assert torch.equal(z, y)


def test_what_lies_between_rows_stays():
    out = torch.full((6, 40), 7.0, device="cuda", dtype=torch.bfloat16)
    layers.layer_norm(torch.randn(6, 33, device="cuda").bfloat16(), out=out[:, :33])
    assert bool((out[:, 33:] == 7.0).all()) and bool((out[:, :33] != 7.0).any())


@pytest.mark.parametrize("rows", [0, 1])
def test_no_rows_give_zero_weight_gradients(rows):
    x, dy = torch.randn(rows, 32, device="cuda"), torch.zeros(rows, 32, device="cuda")
    _, saved = layers.layer_norm(x, save=True)
    dx, dg, db = layers.layer_norm_backward(dy, x, None, saved)
    assert dx.shape == x.shape and not dg.any() and not db.any()


def test_no_rows_of_any_length():
    """Also rows too long for registers, which other kernels take."""
    for c in (32, 2050, 9000, 20001):
        x = torch.empty(0, c, device="cuda")
        y, saved = layers.layer_norm(x, save=True)
        dx, dg, db = layers.layer_norm_backward(y, x, None, saved)
        torch.cuda.synchronize()
        assert dx.shape == x.shape and dg.shape == db.shape == (c,) and not dg.any() and not db.any()


def test_a_constant_row_and_repeated_calls():
    x = torch.full((3, 512), 3.0, device="cuda", dtype=torch.float16)
    y, saved = layers.layer_norm(x, save=True)
    assert not y.any()
    x, dy = (torch.randn(5000, 200, device="cuda").bfloat16() for _ in range(2))
    g = torch.randn(200, device="cuda")
    y, saved = layers.layer_norm(x, g, None, save=True)
    first = layers.layer_norm_backward(dy, x, g, saved)
    for _ in range(3):
        for a, b in zip(first, layers.layer_norm_backward(dy, x, g, saved)):
            assert torch.equal(a, b)


def test_dx_against_differences_of_the_forward_kernel():
    """f32: a central difference with step t has error t^2 |f'''| / 6 + (rounding of
    two losses) / t; both stay below 2e-3 of the largest gradient here."""
    gen = torch.Generator().manual_seed(9)
    x, dy = torch.randn(4, 24, generator=gen).cuda(), torch.randn(4, 24, generator=gen).cuda()
    g, b = torch.randn(24, generator=gen).cuda(), torch.randn(24, generator=gen).cuda()
    _, saved = layers.layer_norm(x, g, b, 1e-2, save=True)
    dx, dg, db = layers.layer_norm_backward(dy, x, g, saved)
    loss = lambda: (layers.layer_norm(x, g, b, 1e-2).double() * dy.double()).sum().item()
    t = 1e-2
    for grad, of in ((dx, x), (dg, g), (db, b)):
        flat = of.view(-1)
        for i in range(0, flat.numel(), 5):
            keep = flat[i].item()
            flat[i] = keep + t
            hi, up = loss(), flat[i].item()
            flat[i] = keep - t
            lo, down = loss(), flat[i].item()
            flat[i] = keep
            diff = (hi - lo) / (up - down)
            assert abs(diff - grad.view(-1)[i].item()) <= 2e-3 * max(1.0, grad.abs().max().item())
