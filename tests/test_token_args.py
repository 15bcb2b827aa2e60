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
