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
