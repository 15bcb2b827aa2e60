"""Refusals and sizes of the token operators, on the host (no GPU needed): every
argument is checked before anything is launched, so the device pointers here
are only numbers."""
import ctypes

import pytest
import torch

from paper_2007_09835_amd import layers, rt3d

A = 1 << 20  # an aligned address that is never followed


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2007_09835_amd import build
    build.build(force=False)


def _status(name, *args):
    lib = rt3d.load()
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    return getattr(lib, name)(*args), lib.rt3d_last_error_detail().decode()


INVALID, UNSUPPORTED, SMALL = (rt3d.RT3D_ERR_INVALID_ARG, rt3d.RT3D_ERR_UNSUPPORTED,
                               rt3d.RT3D_ERR_BUFFER_TOO_SMALL)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(c=0), INVALID), (dict(dtype=7), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x_pitch=7), INVALID),
    (dict(y_pitch=-8), INVALID), (dict(c=(1 << 20) + 1), UNSUPPORTED), (dict(rows=1 << 62), UNSUPPORTED),
])
def test_layer_norm_refuses(change, status):
    d = rt3d.make_norm_desc(4, 8)
    for k, v in change.items():
        setattr(d, k, v)
    got = _status("rt3d_layernorm_fwd", d, A, None, None, A, None, None, None)
    assert got[0] == status and got[1]
    assert _status("rt3d_layernorm_bwd", d, A, A, None, A, A, A, None, None, None, 0, None)[0] == status
    assert _status("rt3d_layernorm_bwd_workspace_size", d, ctypes.byref(ctypes.c_uint64()))[0] == status


def test_layer_norm_pointers():
    d = rt3d.make_norm_desc(4, 8)
    fwd = lambda *a: _status("rt3d_layernorm_fwd", d, *a, None)[0]
    assert fwd(None, None, None, A, None, None) == INVALID
    assert fwd(A, None, None, None, None, None) == INVALID
    assert fwd(A + 1, None, None, A, None, None) == INVALID
    assert fwd(A, A + 2, None, A, None, None) == INVALID
    d.y_pitch = 16
    assert fwd(A, None, None, A, None, None) == INVALID  # in place, two pitches
    d.y_pitch = 0
    assert fwd(A, None, None, A, A + 2, None) == INVALID
    bwd = lambda *a: _status("rt3d_layernorm_bwd", d, *a, None)[0]
    need = rt3d.rt3d_layernorm_bwd_workspace_size(d)
    assert need >= 2 * 8 * 4
    assert bwd(A, None, None, A, A, A, None, None, None, 0) == INVALID
    assert bwd(A, A, None, None, A, A, None, None, None, 0) == INVALID
    assert bwd(A, A, None, A, A, A, A, None, None, 0) == SMALL
    assert bwd(A, A, None, A, A, None, None, A, A, need - 1) == SMALL
    assert bwd(A, A, None, A, A, None, None, None, None, 0) == rt3d.RT3D_OK  # nothing asked for
    d.rows = 0
    assert fwd(None, None, None, None, None, None) == rt3d.RT3D_OK
    assert _status("rt3d_layernorm_fwd", None, A, None, None, A, None, None, None)[0] == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVALID), (dict(t=-1), INVALID), (dict(h=0), INVALID), (dict(w=0), INVALID),
    (dict(vecs=0), INVALID), (dict(d=31), INVALID), (dict(d=0), INVALID), (dict(dt=3), INVALID),
    (dict(dh=-2), INVALID), (dict(dw=24), INVALID), (dict(dtype=-1), INVALID), (dict(flags=4), INVALID),
    (dict(base=0.0), INVALID), (dict(base=float("inf")), INVALID), (dict(t0=-1), INVALID),
    (dict(t0=2 ** 31 - 2), INVALID), (dict(h=1 << 20, w=1 << 20), UNSUPPORTED),
    (dict(x=rt3d.Rows(100, 0)), INVALID), (dict(y=rt3d.Rows(0, -1)), INVALID),
    (dict(y=rt3d.Rows(0, 8)), INVALID),
    (dict(n=2 ** 31 - 1, t=100, vecs=2), UNSUPPORTED),
])
def test_rotation_refuses(change, status):
    d = rt3d.make_rope_desc(2, (3, 2, 2), 4, 32, (8, 12, 12))
    for k, v in change.items():
        setattr(d, k, v)
    got = _status("rt3d_rope3d", d, A, None, A + (1 << 30), None)
    assert got[0] == status and got[1]


def test_rotation_pointers():
    d = rt3d.make_rope_desc(2, (3, 2, 2), 4, 32, (8, 12, 12), y=(160, 0))
    assert _status("rt3d_rope3d", d, None, None, A, None)[0] == INVALID
    assert _status("rt3d_rope3d", d, A, None, None, None)[0] == INVALID
    assert _status("rt3d_rope3d", d, A, A + 2, 2 * A, None)[0] == INVALID
    assert _status("rt3d_rope3d", d, A, None, A, None)[0] == INVALID       # in place, two layouts
    assert _status("rt3d_rope3d", d, A + 1, None, 2 * A, None)[0] == INVALID
    d.t = 0
    assert _status("rt3d_rope3d", d, None, None, None, None)[0] == rt3d.RT3D_OK


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVALID), (dict(lq=-1), INVALID), (dict(lk=-1), INVALID), (dict(hq=0), INVALID),
    (dict(hk=3), INVALID), (dict(hk=0), INVALID), (dict(d=0), INVALID), (dict(d=12), UNSUPPORTED),
    (dict(d=136), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(frame=-1), INVALID),
    (dict(frame=1 << 30), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(lq=1 << 30), UNSUPPORTED), (dict(lk=1 << 30), UNSUPPORTED), (dict(lq=1 << 29), UNSUPPORTED),
    (dict(n=2 ** 31 - 1, lq=64), UNSUPPORTED), (dict(q=rt3d.Rows(100, 0)), INVALID),
    (dict(k=rt3d.Rows(1 << 22, 0)), UNSUPPORTED), (dict(v=rt3d.Rows(132, 0)), UNSUPPORTED),
    (dict(v=rt3d.Rows(0, 12)), UNSUPPORTED), (dict(k=rt3d.Rows(0, -8)), INVALID),
    (dict(o=rt3d.Rows(0, 8)), INVALID),
])
def test_differential_attention_refuses(change, status):
    d = rt3d.make_diffattn_desc(2, 5, 7, 4, 2, 32)
    for k, v in change.items():
        setattr(d, k, v)
    got = _status("rt3d_diffattn_fwd", d, A, A, A, A, None, None, A, None, None, None, 0, None)
    assert got[0] == status and got[1]
    assert _status("rt3d_diffattn_fwd_workspace_size", d, ctypes.byref(ctypes.c_uint64()))[0] == status
    assert _status("rt3d_diffattn_bwd_workspace_size", d, ctypes.byref(ctypes.c_uint64()))[0] == status
    assert _status("rt3d_diffattn_bwd", d, A, A, A, A, None, None, A, A, A, A, A, A, A, A, A, 1 << 40,
                   None)[0] == status


@pytest.mark.parametrize("name", ["dq", "dk", "dv"])
def test_gradients_of_clips_must_not_overlap(name):
    d = rt3d.make_diffattn_desc(2, 5, 7, 4, 2, 32, **{name: (0, 256)})
    assert _status("rt3d_diffattn_bwd_workspace_size", d, ctypes.byref(ctypes.c_uint64()))[0] == INVALID
    assert _status("rt3d_diffattn_fwd_workspace_size", d, ctypes.byref(ctypes.c_uint64()))[0] == rt3d.RT3D_OK


def test_differential_attention_pointers():
    d = rt3d.make_diffattn_desc(2, 5, 7, 4, 2, 32)

    def fwd(**change):
        a = dict(q=A, k=A, v=A, lam=A, ql=None, kl=None, o=A, o2=None, lse=None, ws=None)
        a.update(change)
        return _status("rt3d_diffattn_fwd", d, *a.values(), 0, None)[0]

    for name in ("q", "k", "v", "lam", "o"):
        assert fwd(**{name: None}) == INVALID, name
    for name in ("q", "k", "v", "o", "o2", "ws"):
        assert fwd(**{name: A + 8}) == INVALID, name
    for name in ("lam", "ql", "kl", "lse"):
        assert fwd(**{name: A + 2}) == INVALID, name
    need = rt3d.rt3d_diffattn_bwd_workspace_size(d)

    def bwd(size=need, **change):
        a = dict(q=A, k=A, v=A, lam=A, ql=None, kl=None, o=A, o2=A, lse=A, do=A, dq=A, dk=A, dv=A,
                 dlam=A, ws=A)
        a.update(change)
        return _status("rt3d_diffattn_bwd", d, *a.values(), size, None)[0]

    for name in ("q", "k", "v", "lam", "o", "o2", "lse", "do"):
        assert bwd(**{name: None}) == INVALID, name
    for name in ("q", "k", "v", "o", "o2", "do", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: A + 8}) == INVALID, name
    for name in ("lam", "ql", "kl", "lse", "dlam"):
        assert bwd(**{name: A + 2}) == INVALID, name
    assert bwd(size=need - 1) == SMALL and bwd(ws=None) == SMALL
    assert bwd(dq=None, dk=None, dv=None, dlam=None) == rt3d.RT3D_OK
    d.n = 0
    assert fwd(q=None, k=None, v=None, lam=None, o=None) == rt3d.RT3D_OK


def test_workspaces():
    """Few rows over many keys split, many rows do not; nothing depends on lengths
    on the device."""
    size = lambda *a, **k: rt3d.rt3d_diffattn_fwd_workspace_size(rt3d.make_diffattn_desc(*a, **k))
    assert size(8, 1, 32768, 16, 4, 64) > 0
    assert size(8, 6272, 6272, 16, 4, 64) == 0
    assert size(1, 1, 100, 1, 1, 32) == 0 and size(0, 1, 32768, 1, 1, 32) == 0


def test_the_layers_refuse_what_a_pointer_would_not_show():
    """Shapes, types and strides that the C calls cannot see."""
    t = lambda *s, **k: torch.empty(s, **k)
    with pytest.raises(ValueError, match="gamma"):
        layers.layer_norm(t(4, 8), t(7))
    with pytest.raises(ValueError, match="float32"):
        layers.layer_norm(t(4, 8, dtype=torch.float64))
    with pytest.raises(ValueError, match="beta"):
        layers.layer_norm(t(4, 8), t(8), t(8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="GPU"):
        layers.layer_norm(t(4, 8))
    with pytest.raises(ValueError, match="out"):
        layers.layer_norm(t(4, 8), out=t(4, 9))
    with pytest.raises(ValueError, match="dy"):
        layers.layer_norm_backward(t(3, 8), t(4, 8), None, (t(4), t(4)))
    with pytest.raises(ValueError, match="mean"):
        layers.layer_norm_backward(t(4, 8), t(4, 8), None, (t(3), t(4)))
    with pytest.raises(ValueError, match="grid"):
        layers.rope3d(t(1, 7, 2, 8), (2, 2, 2), (2, 2, 2))
    with pytest.raises(ValueError, match="pos"):
        layers.rope3d(t(1, 8, 2, 8), (2, 2, 2), (2, 2, 2), pos=t(1, 8, 3))
    q, k, v, lam = t(2, 3, 4, 2, 16), t(2, 5, 2, 2, 16), t(2, 5, 2, 32), t(4)
    with pytest.raises(ValueError, match="q must be"):
        layers.diff_attention(q[..., 0, :], k, v, lam)
    with pytest.raises(ValueError, match="k must be"):
        layers.diff_attention(q, k[1:], v, lam)
    with pytest.raises(ValueError, match="v must be"):
        layers.diff_attention(q, k, v.half(), lam)
    with pytest.raises(ValueError, match="lam"):
        layers.diff_attention(q, k, v, t(1))
    with pytest.raises(ValueError, match="k_len"):
        layers.diff_attention(q, k, v, lam, k_len=t(2))
    with pytest.raises(ValueError, match="share memory"):
        layers.diff_attention(q, k[:1].expand(2, 5, 2, 2, 16), v, lam)
    with pytest.raises(ValueError, match="dense"):
        layers.diff_attention(q, k.transpose(3, 4).contiguous().transpose(3, 4), v, lam)
    with pytest.raises(ValueError, match="lse"):
        layers.diff_attention_backward(t(2, 3, 4, 32), q, k, v, lam, (t(2, 3, 4, 32), t(2, 3, 4, 32), t(2, 2, 4, 4)))
    for rows in (t(4, 2, 8).transpose(0, 1), t(8).expand(4, 8)):
        with pytest.raises(ValueError):
            layers._row_pitch(rows, "x")
    assert layers._row_pitch(t(3, 4, 10)[..., :8], "x") == 10


def test_a_scale_of_zero_is_no_default():
    """None asks for 1 / sqrt(d); a number has to be a scale.  An ``out`` of any
    other shape is refused before its strides are looked at."""
    t = torch.empty
    q, k, v, lam = t(2, 3, 4, 2, 16), t(2, 5, 2, 2, 16), t(2, 5, 2, 32), t(4)
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError, match="scale"):
            layers.diff_attention(q, k, v, lam, scale=scale)
    for out in (t(2, 3), t(2, 3, 4, 16), t(2, 3, 4, 32, dtype=torch.float16)):
        with pytest.raises(ValueError, match="out"):
            layers.diff_attention(q, k, v, lam, out=out)


def test_descriptors_hold_the_rows_they_are_given():
    d = rt3d.make_diffattn_desc(1, 2, 3, 4, 2, 16, q=(130, 0), dv=(72, 640))
    assert (d.q.pitch, d.q.batch, d.dv.pitch, d.dv.batch) == (130, 0, 72, 640)
    assert all(r.pitch == r.batch == 0 for r in (d.o, d.k, d.v, d.d_o, d.dq, d.dk))
    r = rt3d.make_rope_desc(1, (1, 2, 3), 2, 8, (2, 2, 2), y=(24, 144))
    assert (r.x.pitch, r.x.batch, r.y.pitch, r.y.batch) == (0, 0, 24, 144)
