"""CPU checks of the 64-bit references that the token operators' GPU tests compare
with: gradients against central differences, the rotation against its inverse."""
import pytest
import torch

import token_refs as refs


def _differences(f, x, step=1e-6):
    g = torch.zeros_like(x)
    flat, out = x.reshape(-1), g.reshape(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + step
        hi = f()
        flat[i] = keep - step
        out[i] = (hi - f()) / (2 * step)
        flat[i] = keep
    return g


def test_layer_norm_gradients_against_differences():
    gen = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(3, 7, generator=gen, dtype=torch.float64) for _ in range(2))
    gamma, beta = (torch.randn(7, generator=gen, dtype=torch.float64) for _ in range(2))
    loss = lambda: (refs.layer_norm(x, gamma, beta, 1e-3)[0] * dy).sum().item()
    _, h, _, rstd = refs.layer_norm(x, gamma, beta, 1e-3)
    for got, of in zip(refs.layer_norm_grads(dy, h, rstd, gamma), (x, gamma, beta)):
        assert torch.allclose(got, _differences(loss, of), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("halves", [False, True])
def test_rotation_is_undone_by_its_inverse_and_keeps_lengths(halves):
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(2, 6, 3, 16, generator=gen, dtype=torch.float64)
    pos = torch.randint(-50, 90000, (2, 6, 3), generator=gen)
    y = refs.rope(x, pos, (4, 6, 2), 1e4, halves, False)
    assert torch.allclose(refs.rope(y, pos, (4, 6, 2), 1e4, halves, True), x, atol=1e-12)
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1))
    assert torch.equal(y[..., 12:], x[..., 12:])


@pytest.mark.parametrize("frame,lens", [(0, None), (1, None), (2, ([4, 3], [3, 5])), (1, ([4, 2], [1, 5]))])
def test_differential_attention_gradients_against_differences(frame, lens):
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)
    q, k, v, lam, do = r(2, 4, 4, 2, 3), r(2, 5, 2, 2, 3), r(2, 5, 2, 6), r(4) * 0.3 + 0.6, r(2, 4, 4, 6)
    ql, kl = (None, None) if lens is None else (torch.tensor(lens[0]), torch.tensor(lens[1]))
    run = lambda: refs.diff_attention(q, k, v, lam, frame, ql, kl)["o"]
    loss = lambda: (run() * do).sum().item()
    got = refs.diff_attention(q, k, v, lam, frame, ql, kl, do=do)
    for name, of in (("dq", q), ("dk", k), ("dv", v), ("dlam", lam)):
        assert torch.allclose(got[name], _differences(loss, of), rtol=1e-5, atol=1e-7), name
    # and the forward pass against torch's softmax, clip by clip
    for b in range(2):
        n_q, n_k = (4, 5) if lens is None else (lens[0][b], lens[1][b])
        for h in range(4):
            o = torch.zeros(4, 6, dtype=torch.float64)
            for i in range(n_q):
                see = refs.visible(i, n_q, n_k, frame)
                if see:
                    p = [torch.softmax(q[b, i, h, m] @ k[b, :see, h // 2, m].T / 3 ** 0.5, -1) for m in (0, 1)]
                    o[i] = (p[0] - lam[h] * p[1]) @ v[b, :see, h // 2]
            assert torch.allclose(run()[b, :, h], o, atol=1e-12)
