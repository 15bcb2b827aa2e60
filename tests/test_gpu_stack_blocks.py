"""Token blocks on every trunk: a trunk's features are what its last layers leave,
eager and in a graph."""
import pytest
import torch

from paper_2007_09835_amd import build, layers, stack

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _features(net):
    """The trunk's last activations, without what its own layers keep beside them."""
    if net.net != "s3d":
        return net.trunk.forward()
    y = net.trunk.forward()
    width = stack.synth.S3D_MIXED[-1]
    return y[..., width[3] + width[5]:]


@pytest.mark.parametrize("name,channels", [("c3d", 512), ("r2plus1d", 512), ("s3d", 1024)])
def test_blocks_on_every_trunk(name, channels):
    net = stack.make_stack(name, batch=1, blocks=2)
    assert [b.c for b in net.blocks] == [channels] * 2
    clips = [torch.rand(net.x.shape, generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i in range(2)]
    eager = []
    for clip in clips:
        net.x.copy_(clip)
        eager.append(net.forward().clone())
        x = _features(net).contiguous()
        assert x.shape[-1] == channels and bool(torch.isfinite(x.float()).all()) and x.any()
        # the same blocks, one after the other, on those features
        for b in net.blocks:
            x = b.forward(x).clone()
        assert torch.equal(x, eager[-1]) and bool(torch.isfinite(x.float()).all())
    assert not torch.equal(eager[0], eager[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.forward()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = net.forward()
    for i in (0, 1, 0):
        net.x.copy_(clips[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i]), i
        net.x.copy_(clips[1 - i])
        assert torch.equal(net.forward(), eager[1 - i])


def test_a_view_of_wider_rows_is_a_block_input():
    b = stack.TokenBlock(64, (2, 3, 5), 2, batch=2)
    row = torch.randn(2, 2, 3, 5, 104, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    x = row[..., 40:]
    want = b.forward(x.contiguous()).clone()
    before = row.clone()
    assert torch.equal(b.forward(x), want) and torch.equal(row, before)
