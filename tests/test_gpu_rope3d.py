"""Rotation by (time, row, column) positions on the GPU against the 64-bit
reference.  A result is a sum of two products: sine and cosine of a turn rounded to
32 bits are off by at most 8 u, the products and their sum add 2 u, the type one
rounding.  The angle itself takes up to 16 roundings of 2^-53 on both sides
(frequency, position times frequency, turns), relative to the position."""
import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


CASES = [
    # n, grid, vecs, d, sections, base
    (1, (1, 1, 1), 1, 2, (2, 0, 0), 1e4), (2, (2, 3, 5), 3, 32, (8, 12, 12), 1e4),
    (3, (4, 7, 7), 16, 64, (16, 24, 24), 1e4), (1, (3, 2, 2), 5, 80, (20, 20, 20), 500.0),
    (2, (2, 4, 4), 4, 18, (6, 6, 2), 1e4), (1, (2, 5, 3), 7, 128, (32, 48, 48), 1e6),
    (2, (3, 3, 1), 2, 24, (0, 12, 8), 1e4), (1, (2, 2, 2), 2, 32, (16, 8, 8), 12345.678901), (1, (9, 28, 28), 32, 64, (16, 24, 24), 1e4),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("given", [False, True])
def test_rotation(case, halves, given, dtype):
    n, grid, vecs, d, sections, base = CASES[case]
    gen = torch.Generator().manual_seed(case)
    tokens = grid[0] * grid[1] * grid[2]
    x, x64 = refs.rounded(torch.randn(n, tokens, vecs, d, generator=gen), dtype)
    pos = torch.randint(-1000, 2 ** 31 - 1, (n, tokens, 3), generator=gen) if given else refs.grid_positions(*grid, t0=77)
    for inverse in (False, True):
        y = layers.rope3d(x.cuda(), grid, sections, base, t0=77, halves=halves, inverse=inverse,
                          pos=pos.to(torch.int32).cuda() if given else None)
        ref = refs.rope(x64, pos, sections, base, halves, inverse)
        size = refs.rope(x64.abs(), pos * 0, sections, base, halves, False)
        pair = torch.zeros_like(size)
        at = 0
        for s in sections:
            for i in range(s // 2):
                a, b = (at + i, at + i + s // 2) if halves else (at + 2 * i, at + 2 * i + 1)
                pair[..., a] = pair[..., b] = size[..., a] + size[..., b]
            at += s
        far = pos.double().abs().amax(-1)[..., None, None] if given else 1000.0
        err = (10 * refs.U + 16 * 2.0 ** -53 * far) * pair
        refs.within(y, ref, err + refs.HALF[dtype] * (ref.abs() + err) + refs.TINY[dtype], "y")
        assert torch.equal(y[..., sum(sections):].cpu(), x[..., sum(sections):])


def test_views_in_place_and_what_is_not_rotated():
    """Queries and keys beside values in one row, rotated where they stand."""
    row = torch.randn(2, 12, 6 * 32, device="cuda").bfloat16()
    before = row.clone()
    qk = row[..., :4 * 32].view(2, 12, 4, 32)
    ref = layers.rope3d(qk.contiguous(), (3, 2, 2), (8, 12, 12))
    assert layers.rope3d(qk, (3, 2, 2), (8, 12, 12), out=qk).data_ptr() == row.data_ptr()
    assert torch.equal(qk, ref)
    assert torch.equal(row[..., 4 * 32:], before[..., 4 * 32:])


@pytest.mark.parametrize("halves", [False, True])
def test_unaligned_views(halves):
    flat = torch.randn(1 + 2 * 6 * 50 + 2, device="cuda").bfloat16()
    x = flat[1:601].view(2, 6, 50)[..., :48].view(2, 6, 2, 24)
    got = layers.rope3d(x, (1, 2, 3), (8, 8, 6), halves=halves)
    assert torch.equal(got, layers.rope3d(x.contiguous(), (1, 2, 3), (8, 8, 6), halves=halves))


def test_infinities_pass_where_nothing_turns():
    x = torch.randn(1, 4, 2, 16, device="cuda")
    x[..., 12:] = float("inf")
    assert bool(torch.isinf(layers.rope3d(x, (1, 2, 2), (4, 4, 4))[..., 12:]).all())


def test_an_empty_batch():
    x = torch.empty(0, 4, 2, 16, device="cuda")
    assert layers.rope3d(x, (1, 2, 2), (4, 4, 4)).shape == x.shape
