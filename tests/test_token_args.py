"""Arguments that the C descriptors would change in silence, and tensors whose
gradient would be lost, on the CPU (nothing is launched)."""
import pytest
import torch

from paper_2007_09835_amd import build, layers, rt3d


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _tensors():
    t = lambda *s: torch.zeros(s)
    return t(2, 3, 4, 2, 16), t(2, 5, 2, 2, 16), t(2, 5, 2, 32), t(4)


def test_tensors_that_want_a_gradient_are_refused():
    """The forward calls leave no autograd graph: they say so, and not by a gradient
    that never comes."""
    x, g, b = torch.zeros(4, 8), torch.ones(8), torch.zeros(8)
    grid = torch.zeros(1, 8, 2, 8)
    calls = [(lambda *a: layers.layer_norm(*a), (x, g, b)),
             (lambda *a: layers.layer_norm(*a, save=True), (x, g, b)),
             (lambda a: layers.rope3d(a, (2, 2, 2), (2, 2, 2)), (grid,)),
             (lambda *a: layers.diff_attention(*a), _tensors()),
             (lambda *a: layers.diff_attention(*a, save=True), _tensors())]
    for call, args in calls:
        for i in range(len(args)):
            wants = [a.clone().requires_grad_(j == i) for j, a in enumerate(args)]
            with pytest.raises(ValueError, match="no_grad"):
                call(*wants)
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):  # as far as a CPU gets
                call(*wants)
            with pytest.raises(ValueError, match="GPU"):
                call(*[a.detach() for a in wants])




@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 64])
def test_numbers_beyond_32_bits_are_refused(big):
    """A descriptor's 32-bit field would keep the low bits: a frame of 2^32 + 5 tokens
    would mask as one of 5."""
    q, k, v, lam = _tensors()
    with pytest.raises(ValueError, match="frame"):
        layers.diff_attention(q, k, v, lam, frame=big)
    with pytest.raises(ValueError, match="frame"):
        layers.diff_attention_backward(torch.zeros(2, 3, 4, 32), q, k, v, lam,
                                       (torch.zeros(2, 3, 4, 32), torch.zeros(2, 3, 4, 32), torch.zeros(2, 2, 4, 3)), frame=big)
    with pytest.raises(ValueError, match="t0"):
        rt3d.make_rope_desc(1, (2, 2, 2), 2, 8, (2, 2, 2), t0=big)
    for i, name in enumerate("thw"):
        grid = [2, 2, 2]
        grid[i] = big
        with pytest.raises(ValueError, match="^%s " % name):
            rt3d.make_rope_desc(1, grid, 2, 8, (2, 2, 2))
    for i, name in enumerate(("dt", "dh", "dw")):
        sections = [2, 2, 2]
        sections[i] = big
        with pytest.raises(ValueError, match=name):
            rt3d.make_rope_desc(1, (2, 2, 2), 2, 8, sections)
    with pytest.raises(ValueError, match="^c "):
        rt3d.make_norm_desc(1, big)
    for i, name in enumerate(("n", "lq", "lk", "hq", "hk", "d")):
        sizes = [1, 2, 3, 4, 2, 16]
        sizes[i] = big
        with pytest.raises(ValueError, match="^%s " % name):
            rt3d.make_diffattn_desc(*sizes)
    for i, name in enumerate(("n", "vecs", "d")):
        sizes = [1, 2, 8]
        sizes[i] = big
        with pytest.raises(ValueError, match="^%s " % name):
            rt3d.make_rope_desc(sizes[0], (2, 2, 2), *sizes[1:], (2, 2, 2))


def test_numbers_at_the_bounds_are_kept():
    d = rt3d.make_diffattn_desc(1, 2 ** 31 - 1, 3, 4, 2, 16, frame=2 ** 31 - 1)
    assert (d.lq, d.frame) == (2 ** 31 - 1,) * 2
    r = rt3d.make_rope_desc(1, (2 ** 31 - 1, 2, 2), 2, 8, (2, 2, 2), t0=-2 ** 31)
    assert (r.t, r.t0) == (2 ** 31 - 1, -2 ** 31)  # (the call then refuses a negative time)
    n = rt3d.make_norm_desc(2 ** 40, 2 ** 31 - 1, x_pitch=2 ** 40)
    assert (n.rows, n.c, n.x_pitch) == (2 ** 40, 2 ** 31 - 1, 2 ** 40)


@pytest.mark.parametrize("scale", [1e-60, 1e39, float("inf")])
def test_a_scale_that_32_bits_do_not_hold(scale):
    """1e-60 would be 0 in the descriptor, which asks for 1 / sqrt(d)."""
    with pytest.raises(ValueError, match="scale"):
        layers.diff_attention(*_tensors(), scale=scale)
