"""What a token block refuses, on the CPU (nothing is launched)."""
import pytest
import torch

from paper_2007_09835_amd import build, stack


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


@pytest.mark.parametrize("c,heads", [(1264, 8), (96, 4), (520, 2), (48, 2)])
def test_heads_that_the_attention_does_not_take(c, heads):
    with pytest.raises(ValueError, match="multiple of 8"):
        stack.TokenBlock(c, (2, 3, 3), heads, device="cpu")


def test_inputs_that_the_pass_would_overwrite():
    """The last conv reads x as its residual while it writes y, and after the other
    buffers have been written."""
    b = stack.TokenBlock(32, (2, 3, 3), 2, batch=2, device="cpu")
    for x in (b.y, b.normed, b.mixed, b.o, b.row[..., :32], b.x.transpose(2, 3), b.y.view(-1).view(b.y.shape)):
        with pytest.raises(ValueError, match="writes"):
            b.stages(x)
    names = [name for name, _ in b.stages()]
    assert names == [name for name, _ in b.stages(b.x)] == [name for name, _ in b.stages(b.y.clone())]
    wide = torch.zeros(2, 2, 3, 3, 40, dtype=b.x.dtype)
    assert [name for name, _ in b.stages(wide[..., 8:])] == ["input"] + names


def test_inputs_that_require_a_gradient():
    """A gathered input must not carry its graph into the block's buffer."""
    b = stack.TokenBlock(32, (2, 3, 3), 2, batch=2, device="cpu")
    wide = torch.zeros(2, 2, 3, 3, 40, dtype=b.x.dtype, requires_grad=True)
    for x in (wide[..., 8:], wide[..., 8:].contiguous()):
        with pytest.raises(ValueError, match="no_grad"):
            b.forward(x)
        assert not b.x.requires_grad
