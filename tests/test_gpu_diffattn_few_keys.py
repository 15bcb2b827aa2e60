"""Gradients of queries that see few keys, on the GPU, against 64 bits.  There the
roundings of o do not average out, so the row sums of P dP must not come from it:
the bound below knows no rounding of o, whatever other rows the call has."""
import math

import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers, rt3d

pytestmark = pytest.mark.gpu

FEW = 32  # every type and size forms the sums of so many keys themselves


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _bounds(q, k, v, do, lam, limit, scale, h, tiny):
    """dq of one clip and query head, [rows][2][d], and the bound on its error: q
    [rows][2][d], k [keys][2][d], v [keys][2 d], do [rows][2 d], limit [rows]."""
    d, kl = q.shape[-1], k.shape[0]
    seen = torch.arange(kl)[None] < limit[:, None]
    dp, dp_size = do @ v.T, do.abs() @ v.abs().T
    dp_err = refs.U * (2 * d + 2) * dp_size
    dq, err = torch.zeros_like(q), torch.zeros_like(q)
    for m, by in ((0, 1.0), (1, -lam)):
        s = (q[:, m] @ k[:, m].T * scale).masked_fill(~seen, -math.inf)
        p = torch.softmax(s, 1)
        size = torch.where(seen, q[:, m].abs() @ k[:, m].abs().T * scale, torch.zeros(()).double())
        # a probability, relatively: its score, exp2, and the logarithm of the
        # denominator, an error of the scores' mean beside its own
        rel = refs.U * ((d + 8) * size + 16 + (kl / 32 + 16))
        perr = rel + rel.max(1, keepdim=True).values
        mean = (p * dp).sum(1, keepdim=True)
        # the sum over 32 keys: its terms' errors and a chain of 48 additions at most
        mean_err = (p * (perr * dp.abs() + dp_err + 48 * refs.U * dp.abs())).sum(1, keepdim=True)
        ds = by * p * (dp - mean) * scale
        e = abs(by) * scale * p * ((perr + h + 3 * refs.U) * (dp - mean).abs() + (1 + h) * (dp_err + mean_err))
        e = e + scale * tiny * max(1.0, abs(by)) * seen
        dq[:, m] = ds @ k[:, m]
        e = (e + refs.U * (kl + 8) * ds.abs()) @ k[:, m].abs()
        err[:, m] = e + max(h, refs.U) * (dq[:, m].abs() + e) + tiny * 4 + 1e-30
    return dq, err


def _inputs(n, lq, lk, hq, hk, d, dtype):
    gen = torch.Generator().manual_seed(lq + lk + d)
    r = lambda *s: torch.randn(s, generator=gen)
    # values and output gradients off zero: o and its roundings are large beside dP - A
    return (refs.rounded(r(n, lq, hq, 2, d), dtype), refs.rounded(r(n, lk, hk, 2, d), dtype),
            refs.rounded(r(n, lk, hk, 2 * d) + 3.0, dtype), refs.rounded(r(n, lq, hq, 2 * d), dtype),
            r(hq) * 0.2 + 0.6)


def _run(q, k, v, do, lam, **more):
    args = [t[0].cuda() for t in (q, k, v)] + [lam.cuda()]
    _, saved = layers.diff_attention(*args, save=True, **more)
    return layers.diff_attention_backward(do[0].cuda(), *args, saved, **more)


CASES = [(2, 200, 200, 2, 2), (1, 700, 700, 4, 1), (2, 150, 90, 2, 1), (1, 1100, 1100, 1, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("frame", [1, 5])
@pytest.mark.parametrize("n,lq,lk,hq,hk", CASES)
def test_early_rows_of_causal_calls(n, lq, lk, hq, hk, frame, d, dtype):
    """Rows of 1 to 32 keys in calls whose other rows see many; split and not."""
    q, k, v, do, lam = _inputs(n, lq, lk, hq, hk, d, dtype)
    got = _run(q, k, v, do, lam, frame=frame)[0]
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    limit = torch.tensor([refs.visible(i, lq, lk, frame) for i in range(lq)])
    rows = ((limit > 0) & (limit <= FEW)).nonzero()[:, 0]
    for b in range(n):
        for head in range(hq):
            kv = head // (hq // hk)
            # (the softmax of a single key does not move)
            ref, err = _bounds(q[1][b, rows, head], k[1][b, :FEW, kv], v[1][b, :FEW, kv], do[1][b, rows, head],
                               float(lam[head]), limit[rows], 1 / math.sqrt(d), h, refs.TINY[dtype])
            ref[limit[rows] == 1] = 0.0
            refs.within(got[b, rows, head], ref, err, f"dq clip {b} head {head}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_short_clips_beside_long_ones(d, dtype):
    """A clip of a few keys in a call whose other clips' keys are split."""
    n, lq, lk, hq, hk = 3, 100, 400, 2, 1
    q, k, v, do, lam = _inputs(n, lq, lk, hq, hk, d, dtype)
    lens = [400, 3, 32]
    got = _run(q, k, v, do, lam, k_len=torch.tensor(lens, dtype=torch.int32).cuda())
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    for b in (1, 2):
        for head in range(hq):
            ref, err = _bounds(q[1][b, :, head], k[1][b, :lens[b], 0], v[1][b, :lens[b], 0], do[1][b, :, head],
                               float(lam[head]), torch.full((lq,), lens[b]), 1 / math.sqrt(d), h, refs.TINY[dtype])
            refs.within(got[0][b, :, head], ref, err, f"dq clip {b} head {head}")


@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (64, "f16"), (128, "bf16"), (64, "f32")])
def test_a_clip_alone_and_beside_longer_ones(d, dtype):
    """dk of a short clip: the same sums reach it whatever else its call has, so it
    is what the clip alone gives, within the order of its sums (and one rounding)."""
    lq, lk, hq, hk = 100, 400, 2, 1
    q, k, v, do, lam = _inputs(2, lq, lk, hq, hk, d, dtype)
    both = _run(q, k, v, do, lam, k_len=torch.tensor([400, 3], dtype=torch.int32).cuda())
    pick = lambda t, keys: (t[0][1:, :3].contiguous() if keys else t[0][1:], None)
    alone = _run(pick(q, 0), pick(k, 1), pick(v, 1), pick(do, 0), lam)
    assert rt3d.rt3d_diffattn_bwd_workspace_size(rt3d.make_diffattn_desc(2, lq, lk, hq, hk, d, dtype)) > 0
    step = torch.finfo(refs.TDT[dtype]).eps
    for a, b in zip(both[:2], alone[:2]):
        a, b = a[1, :b.shape[1]].double(), b[0].double()
        # the two calls' probabilities are the same but for their reference (exp2 and
        # its logarithm, 2^-20), so dS is the same but for a few that round the other way
        size = b.abs() + b.abs().amax()
        assert ((a - b).abs() <= step * size + 2.0 ** -20 * size).all()
