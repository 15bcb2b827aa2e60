"""The token operators run together, as they are used: a token block on a conv
trunk's features, stage by stage against 64 bits and captured in HIP graphs, and a
training step through layer norm, rotation and differential attention."""
import numpy as np
import pytest
import torch

import token_refs as refs
from harness import error_bound
from paper_2007_09835_amd import build, layers, stack

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _conv_check(x, w, b, res, y, dtype, label):
    """A 1x1x1 conv within the conv kernels' per-output bound."""
    c = x.shape[-1]
    x64, w64 = x.double().cpu().reshape(-1, c), w.double().reshape(w.shape[0], c)
    b64 = torch.from_numpy(b).double()
    ref, size = x64 @ w64.T + b64, x64.abs() @ w64.abs().T + b64.abs()
    if res is not None:
        r = res.double().cpu().reshape(ref.shape)
        ref, size = ref + r, size + r.abs()
    bound = torch.from_numpy(error_bound(ref.numpy(), size.numpy(), c, dtype))
    refs.within(y.reshape(ref.shape), ref, bound, label)


@pytest.mark.parametrize("dtype,causal,heads,key_heads", [("bf16", False, 4, None), ("f16", True, 8, 2), ("f32", True, 2, 1)])
def test_block_stage_by_stage(dtype, causal, heads, key_heads):
    """Every stage against 64 bits on what the stage before it left on the GPU."""
    n, thw, c = 2, (3, 5, 4), 128
    b = stack.TokenBlock(c, thw, heads, key_heads, n, dtype, causal, depth=2)
    b.x.copy_(torch.randn(b.x.shape, generator=torch.Generator().manual_seed(1)) + 0.5)
    stages = dict(b.stages())
    half, u = refs.HALF[dtype], refs.U
    stages["norm"]()
    norm = lambda x, g, be, y, label: _norm_check(x, g, be, y, dtype, label)
    norm(b.x, b.gamma, b.beta, b.normed, "norm")
    stages["qkv"]()
    _conv_check(b.normed, b.w_qkv, b.b_qkv, None, b.row, dtype, "qkv")
    before = b.turned.double().cpu()
    values = b.v.clone()
    stages["rope"]()
    ref = refs.rope(before, refs.grid_positions(*thw), b.sections, 1e4, False, False)
    bound = 12 * u * before.abs().amax(-1, keepdim=True) * 2
    refs.within(b.turned, ref, bound + half * (ref.abs() + bound) + refs.TINY[dtype], "rope")
    assert torch.equal(values, b.v)
    stages["attention"]()
    got = refs.diff_attention(b.q.double().cpu(), b.k.double().cpu(), b.v.double().cpu(), b.lam.double().cpu(),
                              b.frame, h=0.0 if dtype == "f32" else half, tiny=refs.TINY[dtype])
    o = b.o.view(n, b.tokens, heads, 2 * b.d)
    refs.within(o, got["o"], got["o_err"] + u * got["o"].abs() + 4 * refs.TINY[dtype] + 1e-30, "attention")
    stages["head_norm"]()
    norm(b.o.view(-1, 2 * b.d), b.head_gamma, b.head_beta, b.mixed.view(-1, 2 * b.d), "head_norm")
    stages["proj"]()
    _conv_check(b.mixed, b.w_out, b.b_out, b.x, b.y, dtype, "proj")
    y = b.y.clone()
    assert torch.equal(b.forward(), y)


def _norm_check(x, g, be, y, dtype, label):
    c = x.shape[-1]
    x64, g64, b64 = x.double().cpu().reshape(-1, c), g.double().cpu(), be.double().cpu()
    ref, h, _, rstd = refs.layer_norm(x64, g64, b64, 1e-5)
    bound = refs.norm_h_error(x64, h, rstd, c) * g64.abs() + 3 * refs.U * (h.abs() * g64.abs() + b64.abs())
    refs.within(y.reshape(-1, c), ref, bound + refs.HALF[dtype] * (ref.abs() + bound) + refs.TINY[dtype], label)


def _captured(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


def test_trunk_and_blocks_in_a_graph():
    """C3D with two token blocks, captured; replays with new clips, with the eager
    pass and another graph between them, repeat the eager results."""
    net = stack.make_stack("c3d", batch=2, blocks=2)
    other = stack.TokenBlock(64, (2, 3, 3), 2, batch=1)
    clips = [torch.rand(net.x.shape, generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i in range(3)]
    eager = []
    for clip in clips:
        net.x.copy_(clip)
        eager.append(net.forward().clone())
    assert not torch.equal(eager[0], eager[1]) and bool(torch.isfinite(eager[0].float()).all())
    graph, second = _captured(net.forward), _captured(other.forward)
    for i in (0, 1, 2, 1, 0):
        net.x.copy_(clips[i])
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        assert torch.equal(net.blocks[-1].y, eager[i]), i
        net.x.copy_(clips[(i + 1) % 3])
        assert torch.equal(net.forward(), eager[(i + 1) % 3])


def _train_step(x, w, gamma, beta, lam, dy, thw, heads, sections, frame):
    """Loss gradient of sum(o dy) through norm, a product with w, rotation and
    attention, by the library's backward calls (the products are torch's)."""
    n, tokens, c = x.shape
    d = c // (2 * heads)
    u, saved = layers.layer_norm(x, gamma, beta, save=True)
    row = torch.matmul(u.view(-1, c), w).view(n, tokens, 3 * c)
    qk = layers.rope3d(row[..., :2 * c].view(n, tokens, 4 * heads, d), thw, sections)
    q, k = qk[:, :, :2 * heads].view(n, tokens, heads, 2, d), qk[:, :, 2 * heads:].view(n, tokens, heads, 2, d)
    v = row[..., 2 * c:].view(n, tokens, heads, 2 * d)
    o, kept = layers.diff_attention(q, k, v, lam, frame, save=True)
    dq, dk, dv, dlam = layers.diff_attention_backward(dy, q, k, v, lam, kept, frame)
    dqk = torch.cat([dq.view(n, tokens, 2 * heads, d), dk.view(n, tokens, 2 * heads, d)], 2)
    layers.rope3d(dqk, thw, sections, inverse=True, out=dqk)
    drow = torch.cat([dqk.view(n, tokens, 2 * c), dv.reshape(n, tokens, c)], 2).view(-1, 3 * c)
    dw = torch.matmul(u.view(-1, c).t().contiguous(), drow)
    du = torch.matmul(drow, w.t().contiguous()).view(n, tokens, c)
    return (o, *layers.layer_norm_backward(du, x, gamma, saved), dw, dlam)


def test_a_training_step_against_64_bit_autograd():
    """float32: about a dozen stages, each off by the accumulation of up to 3 c
    products (relative 2-norm far below 1e-5 each, random signs), a softmax that
    carries scores' errors with a factor of a few: 1e-4 holds them all."""
    n, thw, heads, c = 2, (2, 4, 5), 2, 64
    tokens, d, sections, frame = 40, 16, (4, 6, 6), 20
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen)
    x, w, gamma, beta = r(n, tokens, c), r(c, 3 * c) / 8, 1 + 0.1 * r(c), 0.1 * r(c)
    lam, dy = 0.6 + 0.1 * r(heads), r(n, tokens, heads, 2 * d)
    got = _train_step(*(t.cuda() for t in (x, w, gamma, beta, lam, dy)), thw, heads, sections, frame)
    X, W, G, B, L = (t.double().requires_grad_() for t in (x, w, gamma, beta, lam))
    u = refs.layer_norm(X.view(-1, c), G, B, 1e-5)[0]
    row = (u @ W).view(n, tokens, 3 * c)
    pos = refs.grid_positions(*thw)
    qk = row[..., :2 * c].view(n, tokens, 4 * heads, d)
    parts, at = [], 0
    for axis, size in enumerate(sections):
        i = torch.arange(size // 2)
        th = pos[..., axis:axis + 1].double() * 1e4 ** (-2.0 * i / size)
        a, b = qk[..., at:at + size:2], qk[..., at + 1:at + size:2]
        cs, sn = torch.cos(th)[:, :, None], torch.sin(th)[:, :, None]
        parts.append(torch.stack([a * cs - b * sn, a * sn + b * cs], -1).flatten(-2))
        at += size
    qk = torch.cat(parts, -1)
    q, k = (t.reshape(n, tokens, heads, 2, d) for t in qk.split(2 * heads, 2))
    s = torch.einsum("iahmd,ibhmd->ihmab", q, k) / d ** 0.5
    f = torch.arange(tokens) // frame
    p = torch.softmax(s.masked_fill(f[None] > f[:, None], float("-inf")), -1)
    mix = p[:, :, 0] - L.view(1, heads, 1, 1) * p[:, :, 1]
    o = torch.einsum("ihab,ibhe->iahe", mix, row[..., 2 * c:].view(n, tokens, heads, 2 * d))
    o.backward(dy.double())
    for name, a, b in zip(("o", "dx", "dgamma", "dbeta", "dw", "dlam"), got,
                          (o.detach(), X.grad, G.grad, B.grad, W.grad, L.grad)):
        rel = ((a.double().cpu() - b).norm() / b.norm()).item()
        print(f"{name}: relative 2-norm {rel:.2e}", flush=True)
        assert rel <= 1e-4, (name, rel)


def test_a_training_step_in_a_graph():
    """Forward and backward captured together, replayed with eager steps on the same
    tensors between; every replay equals the eager result."""
    n, thw, heads, c = 2, (3, 7, 7), 2, 128
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(s, generator=gen).cuda()
    lam, dy = 0.6 + 0.1 * r(heads), r(n, 147, heads, c // heads).bfloat16()
    x, gamma, beta = r(n, 147, c).bfloat16(), 1 + 0.1 * r(c), 0.1 * r(c)
    row = r(n, 147, 3 * c).bfloat16()
    out = {}

    def step():
        u, saved = layers.layer_norm(x, gamma, beta, save=True)
        view = lambda i: (row[..., i * c:(i + 1) * c]).view(n, 147, heads, -1)
        q, k = (layers.rope3d(view(i).view(n, 147, 2 * heads, 32), thw, (8, 12, 12)).view(n, 147, heads, 2, 32)
                for i in (0, 1))
        o, kept = layers.diff_attention(q, k, view(2), lam, 49, save=True)
        grads = layers.diff_attention_backward(dy, q, k, view(2), lam, kept, 49)
        out["all"] = (u, o, *grads, *layers.layer_norm_backward(dy.view(n, 147, c), x, gamma, saved))

    step()
    want = [t.clone() for t in out["all"]]
    graph = _captured(step)
    captured = out["all"]
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b)
        x.mul_(1.5)
        row.mul_(0.75)
        step()
        want = [t.clone() for t in out["all"]]


def test_two_streams_at_once():
    """Two blocks on two streams give what they give alone."""
    a, b = stack.TokenBlock(64, (4, 7, 7), 2, tag="a"), stack.TokenBlock(128, (2, 9, 9), 2, 1, causal=True, tag="b")
    for i, blk in enumerate((a, b)):
        blk.x.copy_(torch.randn(blk.x.shape, generator=torch.Generator().manual_seed(i)))
    alone = [blk.forward().clone() for blk in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for blk, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                blk.y.zero_()
                blk.forward()
    torch.cuda.synchronize()
    assert torch.equal(a.y, alone[0]) and torch.equal(b.y, alone[1])
