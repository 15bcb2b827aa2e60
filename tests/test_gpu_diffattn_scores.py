"""Differential attention on the GPU where scores are -inf or rise along the keys:
the reference that a row's probabilities are formed against has to be found late,
or moved.  Against 64 bits, within the bounds that token_refs derives."""
import math

import pytest
import torch

import token_refs as refs
from paper_2007_09835_amd import build, layers, rt3d

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build(force=False)


def _inputs(seed, n, lq, lk, hq, hk, d, dtype):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    q = refs.rounded(r(n, lq, hq, 2, d), dtype)
    k = refs.rounded(r(n, lk, hk, 2, d), dtype)
    v = refs.rounded(r(n, lk, hk, 2 * d) + 0.3, dtype)
    do = refs.rounded(r(n, lq, hq, 2 * d), dtype)
    return q, k, v, do, r(hq) * 0.2 + 0.6


def _hide(q, k, hidden, big):
    """Channel 0 of map m makes the scores of the keys in hidden[m] -inf (``big``: as
    a product of finite numbers, 2^-84 and 2^84) and adds nothing elsewhere."""
    for qq, kk in zip(q, k):
        qq[..., 0] = 2.0 ** 84 if big else 1.0
        kk[..., 0] = 0.0
        for m in (0, 1):
            kk[:, hidden[m], :, m, 0] = -2.0 ** 84 if big else -math.inf


def _without(q, k, v, lam, hidden, dtype, **more):
    """o, o2 and lse of every map over the keys that it has left, and their bounds."""
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    maps = []
    for m in (0, 1):
        left = ~hidden[m]
        kk = k[1][:, left].clone()
        if hidden[1 - m].any():
            kk[..., 1 - m, 0] = 0.0  # (the other map's results are not used)
        maps.append(refs.diff_attention(q[1], kk, v[1][:, left], lam.double() * m, h=h, tiny=refs.TINY[dtype], **more))
    l = lam.double().view(1, 1, -1, 1)
    half = refs.U if dtype == "f32" else h
    o, o2 = maps[0]["o"] - l * maps[1]["o2"], maps[1]["o2"]
    o_err = maps[0]["o_err"] + l * maps[1]["o2_err"]
    tiny = refs.TINY[dtype] * 4 + 1e-30
    return (o, o_err + half * (o.abs() + o_err) + tiny, o2, maps[1]["o2_err"] + half * o2.abs() + tiny,
            torch.stack([maps[0]["lse"][0], maps[1]["lse"][1]]))


def _forward_check(q, k, v, lam, hidden, dtype, scale=None, far=64.0):
    """``far``: what no score (times log2 e) exceeds."""
    n, lq, hq, _, d = q[0].shape
    lk, hk = k[0].shape[1:3]
    args = [t[0].cuda() for t in (q, k, v)] + [lam.cuda()]
    o_ref, o_err, o2_ref, o2_err, lse_ref = _without(q, k, v, lam, hidden, dtype, scale=scale)
    desc = rt3d.make_diffattn_desc(n, lq, lk, hq, hk, d, dtype, scale=scale or 0.0)
    for name in ("workspace", "none"):
        o = torch.empty(n, lq, hq, 2 * d, dtype=args[0].dtype, device="cuda")
        o2, lse = torch.empty_like(o), torch.empty(2, n, hq, lq, device="cuda")
        ws = None
        if name == "workspace":
            ws = torch.empty(rt3d.rt3d_diffattn_fwd_workspace_size(desc) // 4, device="cuda")
        rt3d.rt3d_diffattn_fwd(desc, *args, None, None, o, o2, lse, ws)
        refs.within(o, o_ref, o_err, f"o, {name}")
        refs.within(o2, o2_ref, o2_err, f"o2, {name}")
        seen = torch.isfinite(lse_ref)
        got = lse.double().cpu()
        assert torch.equal(torch.isfinite(got), seen)
        # a score's error, d + 8 roundings of it, and 2^-11 for the sum and its logarithm
        assert ((got - lse_ref)[seen].abs() <= far * (d + 8) * refs.U + 2.0 ** -11).all()
        assert (got[~seen] == math.inf).all()


def _masks(lk, kind):
    j = torch.arange(lk)
    none = j < 0
    return {"first": (j < 40, j < 32), "one map": (none, j < 33), "blocks": (j // 32 % 3 == 0, j // 64 % 2 == 0),
            "a split": ((j >= 512) & (j < 1100), j // 32 % 2 == 0), "all of one": (none, ~none),
            "all of the other": (~none, j < 7), "all but the last": (j < lk - 1, j < lk - 2)}[kind]


KINDS = ["first", "one map", "blocks", "a split", "all of one", "all of the other", "all but the last"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lq,lk", [(1, 2100), (40, 1300)])
@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "f16"), (128, "bf16"), (64, "f32"), (96, "f32")])
def test_keys_hidden_by_a_channel(d, dtype, lq, lk, kind):
    """A key channel of -inf hides a key from every query, split and unsplit: at the
    start of a clip, of a split, or everywhere."""
    q, k, v, _, lam = _inputs(5, 1, lq, lk, 2, 1, d, dtype)
    hidden = _masks(lk, kind)
    _hide(q, k, hidden, False)
    _forward_check(q, k, v, lam, hidden, dtype)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_the_keys_left_score_far_below_zero(d):
    """Formed against 0, every probability would vanish."""
    q, k, v, _, lam = _inputs(6, 1, 33, 200, 1, 1, d, "bf16")
    hidden = _masks(200, "first")
    _hide(q, k, hidden, False)
    for qq, kk in zip(q, k):
        qq[..., 1], kk[..., 1] = 64.0, -64.0
    _forward_check(q, k, v, lam, hidden, "bf16", scale=1.0, far=8192.0)


@pytest.mark.parametrize("lq,lk", [(70, 200), (33, 900)])
@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (128, "bf16"), (64, "f32")])
def test_gradients_where_scores_pass_the_range(d, dtype, lq, lk):
    """Finite queries and keys whose product is -inf in 32 bits: such keys get no
    gradient, the others theirs."""
    q, k, v, do, lam = _inputs(7, 2, lq, lk, 2, 1, d, dtype)
    one = torch.arange(lk) < 37
    _hide(q, k, (one, one), True)
    args = [t[0].cuda() for t in (q, k, v)] + [lam.cuda()]
    o, saved = layers.diff_attention(*args, save=True)
    grads = layers.diff_attention_backward(do[0].cuda(), *args, saved)
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    ref = refs.diff_attention(q[1], k[1][:, ~one], v[1][:, ~one], lam.double(), do=do[1], h=h, tiny=refs.TINY[dtype])
    half, tiny = refs.U if dtype == "f32" else 0.0, refs.TINY[dtype] * 4 + 1e-30
    refs.within(o, ref["o"], ref["o_err"] + half * ref["o"].abs() + tiny, "o")
    for name, got in zip(("dq", "dk", "dv", "dlam"), grads):
        if name in ("dk", "dv"):
            assert not got[:, :37].any()
            got = got[:, 37:]
        refs.within(got, ref[name], ref[name + "_err"] + half * ref[name].abs() + tiny, name)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "f16"), (128, "bf16"), (128, "f16"), (64, "f32"), (96, "f32")])
@pytest.mark.parametrize("lq,lk", [(33, 700), (200, 300), (1, 3000)])
def test_scores_that_rise_along_the_keys(d, dtype, lq, lk):
    """One map's scores rise by 160 over the keys, so that every second step of 32 or
    so starts again with a new reference; the other's fall.  Beyond d 32, where the
    values' loads and the maps are dealt out otherwise."""
    q, k, v, _, lam = _inputs(31, 1, lq, lk, 1, 1, d, dtype)
    ramp = torch.linspace(0, 20, lk)
    for m, by in ((0, ramp), (1, -ramp)):
        kk, qq = k[0], q[0]
        kk[0, :, 0, m, 0], qq[0, :, 0, m, 0] = by.to(kk.dtype), 8.0
    for t in (q, k):
        t[1].copy_(t[0].double())
    none = torch.zeros(lk, dtype=torch.bool)
    _forward_check(q, k, v, lam, (none, none), dtype, scale=1.0, far=512.0)


@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (128, "bf16"), (64, "f32"), (96, "f32")])
@pytest.mark.parametrize("lq,lk", [(33, 500), (70, 200), (30, 2100)])
def test_rows_that_wait_for_a_score_beside_rows_that_rise(d, dtype, lq, lk):
    """Every other row has scores of -inf for 150 keys; the scores of those between
    rise by 160 nats over them, far past the range of a probability."""
    q, k, v, _, lam = _inputs(8, 1, lq, lk, 1, 1, d, dtype)
    late = torch.arange(lk) < 150
    ramp = torch.linspace(0, 20, 150)
    for qq, kk in zip(q, k):
        qq[..., :2] = 0.0
        kk[..., :2] = 0.0
        qq[:, ::2, ..., 0] = 2.0 ** 84
        kk[:, late, ..., 0] = -2.0 ** 84
        qq[:, 1::2, ..., 1] = 8.0
        kk[:, late, ..., 1] = ramp.to(k[0].dtype).to(kk.dtype).view(1, 150, 1, 1)
    o = layers.diff_attention(q[0].cuda(), k[0].cuda(), v[0].cuda(), lam.cuda(), scale=1.0)
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    more = dict(scale=1.0, h=h, tiny=refs.TINY[dtype])
    half, tiny = refs.U if dtype == "f32" else 0.0, refs.TINY[dtype] * 4 + 1e-30
    for rows, keys in ((slice(0, None, 2), ~late), (slice(1, None, 2), late | ~late)):
        qq, kk = q[1][:, rows].contiguous(), k[1][:, keys].clone()
        kk[..., 0] = 0.0
        qq[..., 0] = 0.0
        ref = refs.diff_attention(qq, kk, v[1][:, keys], lam.double(), **more)
        refs.within(o[:, rows], ref["o"], ref["o_err"] + half * ref["o"].abs() + tiny, "o")


@pytest.mark.parametrize("lq,lk,q_len", [(70, 200, None), (33, 900, None), (64, 200, [64, 40]), (128, 300, [1, 0])])
@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "f16"), (128, "bf16"), (64, "f32"), (96, "f32")])
def test_gradients_beside_hidden_keys(d, dtype, lq, lk, q_len):
    """Keys hidden by a channel of -inf get no gradient and change nobody's, whatever
    rows lie behind the clip's last query: only dq's own channel, 0 times -inf, is NaN."""
    q, k, v, do, lam = _inputs(9, 2, lq, lk, 2, 1, d, dtype)
    hidden = torch.arange(lk) // 8 % 3 == 1
    _hide(q, k, (hidden, hidden), False)
    args = [t[0].cuda() for t in (q, k, v)] + [lam.cuda()]
    more = dict(q_len=None if q_len is None else torch.tensor(q_len, dtype=torch.int32).cuda())
    _, saved = layers.diff_attention(*args, save=True, **more)
    grads = layers.diff_attention_backward(do[0].cuda(), *args, saved, **more)
    h = 0.0 if dtype == "f32" else refs.HALF[dtype]
    ref = refs.diff_attention(q[1], k[1][:, ~hidden], v[1][:, ~hidden], lam.double(), 0, q_len, do=do[1], h=h,
                              tiny=refs.TINY[dtype])
    half, tiny = refs.U if dtype == "f32" else 0.0, refs.TINY[dtype] * 4 + 1e-30
    for name, got in zip(("dq", "dk", "dv", "dlam"), grads):
        want, err = ref[name], ref[name + "_err"]
        if name in ("dk", "dv"):
            assert not got[:, hidden].any(), name
            got = got[:, ~hidden]
        if name == "dq":
            got, want, err = got[..., 1:], want[..., 1:], err[..., 1:]
        refs.within(got, want, err + half * want.abs() + tiny, name)
