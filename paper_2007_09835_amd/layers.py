"""Layer objects over the C ABI: pack once on the host, keep the blob and
bias on the device, launch the HIP kernels per call.

Memory management and argument marshalling only; every arithmetic step of a
forward pass runs in librt3d's kernels.  Activations are channels-last
contiguous device tensors [n, t, h, w, c].
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np
import torch

from . import rt3d

TORCH_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Conv3d:
    """One packed 3-D convolution (dense when ``mask`` is None, else KGS).

    ``w`` is a host tensor [M][N][kt][kh][kw] already in the layer dtype;
    ``bias`` a host float array [M] (or None); ``mask`` uint8 [P][Q][K_s].
    """

    def __init__(self, c_in: int, c_out: int, thw: Sequence[int], k, stride, pad, w,
                 bias=None, mask: Optional[np.ndarray] = None, dtype: str = "bf16",
                 relu: bool = True, residual: bool = False, g=(4, 4), device="cuda",
                 batch: int = 1, pool=(1, 1, 1)):
        """``batch`` is the batch size the layer is planned for (the blob
        works for any batch; the tile shapes are chosen for this one).
        ``pool`` fuses a max-pool (window = stride) after the activation."""
        self.dtype = dtype
        self.sparse = mask is not None
        self.desc = rt3d.make_desc(batch, c_in, c_out, tuple(thw), tuple(k), tuple(stride),
                                   tuple(pad), tuple(g), dtype, relu=relu, residual=residual,
                                   pool=tuple(pool))
        if self.sparse:
            blob, self.info = rt3d.rt3d_kgs_pack(self.desc, w, mask)
        else:
            blob, self.info = rt3d.rt3d_dense_pack(self.desc, w)
        self.blob = torch.from_numpy(blob).to(device)
        self.bias = None if bias is None else torch.as_tensor(
            np.asarray(bias, dtype=np.float32)).to(device)
        self.out_thw = rt3d.rt3d_conv3d_out_shape(self.desc)
        self.c_out = c_out
        self.device = device
        self._ws = {}

    def desc_for(self, n: int) -> rt3d.Conv3dDesc:
        d = rt3d.Conv3dDesc.from_buffer_copy(self.desc)
        d.n = n
        return d

    def out_shape(self, n: int):
        return (n, *self.out_thw, self.c_out)

    def workspace(self, n: int) -> Optional[torch.Tensor]:
        """Split-K workspace for batch n (allocated once per batch size)."""
        if n not in self._ws:
            nbytes = rt3d.rt3d_conv3d_workspace_size(self.desc_for(n), self.info)
            self._ws[n] = (None if nbytes == 0 else
                           torch.empty(nbytes // 4, dtype=torch.float32, device=self.device))
        return self._ws[n]

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stream=None,
                 use_workspace: bool = True, c_off: int = 0, x_off: int = 0) -> torch.Tensor:
        """``out`` may hold more channels than c_out: the layer then writes
        channels [c_off, c_off + c_out) of it (fused concatenation); ``x``
        may hold more channels than c_in: the layer reads [x_off, x_off +
        c_in) of it."""
        n = x.shape[0]
        if out is None:
            out = torch.empty(self.out_shape(n), dtype=TORCH_DTYPES[self.dtype], device=x.device)
        ws = self.workspace(n) if use_workspace and n > 0 else None
        d = self.desc_for(n)
        if out.shape[-1] != self.c_out or c_off:
            d.y_c_total, d.y_c_off = out.shape[-1], c_off
        if x.shape[-1] != d.c_in or x_off:
            d.x_c_total, d.x_c_off = x.shape[-1], x_off
        fwd = rt3d.rt3d_kgs_conv3d_fwd if self.sparse else rt3d.rt3d_conv3d_dense_fwd
        fwd(d, self.info, self.blob, x, self.bias, residual, out, ws, stream)
        return out


def maxpool3d(x: torch.Tensor, k, stride, dtype: str, out: Optional[torch.Tensor] = None,
              stream=None, pad=(0, 0, 0)) -> torch.Tensor:
    n, t, h, w, c = x.shape
    to, ho, wo = ((t + 2 * pad[0] - k[0]) // stride[0] + 1, (h + 2 * pad[1] - k[1]) // stride[1] + 1,
                  (w + 2 * pad[2] - k[2]) // stride[2] + 1)
    if out is None:
        out = torch.empty((n, to, ho, wo, c), dtype=x.dtype, device=x.device)
    rt3d.rt3d_maxpool3d_fwd(x, out, k, stride, dtype, stream, pad)
    return out


# ---------------------------------------------------------------------------
# Token operators
#
# Inputs are tensors whose last dimension is dense; views into wider rows (a
# projection's queries beside its keys, the filled part of a cache) are taken as
# they are.  Results are new tensors unless ``out`` is given, which may be x itself in
# layer_norm and rope3d and must not overlap an input otherwise.  A call runs on the
# device of its tensors, on ``stream`` (a torch stream of that device) or else on
# that device's current stream; its results and workspace belong to that stream.
# Gradients come from the backward calls; results carry no autograd graph, so with
# gradients enabled the forward calls refuse tensors that require one.
# ---------------------------------------------------------------------------

_CODES = {dt: name for name, dt in TORCH_DTYPES.items()}


def _dtype_of(x: torch.Tensor, name: str) -> str:
    if x.dtype not in _CODES:
        raise ValueError("%s must be float32, bfloat16 or float16, not %s" % (name, x.dtype))
    return _CODES[x.dtype]


def _need(t: Optional[torch.Tensor], name: str, like: torch.Tensor, shape, dtype) -> None:
    """``t`` (if there is one) lies on ``like``'s device with this shape and type."""
    if t is None:
        return
    if t.device != like.device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, like.device))
    if t.dtype != dtype:
        raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.shape != shape:  # a torch.Size is a tuple
        raise ValueError("%s must be %s, not %s" % (name, list(shape), list(t.shape)))


def _no_graph(*tensors) -> None:
    """Refuses tensors whose gradient would be lost: the results carry no graph."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("a tensor requires a gradient, and the result would carry none: call under "
                                 "torch.no_grad() and take gradients from the backward call")


def _launch(x: torch.Tensor, stream, call):
    """``call()`` with ``x``'s device and ``stream`` current."""
    if not x.is_cuda:
        raise ValueError("tensors must be on a GPU")
    if stream is not None:
        if stream.device != x.device:
            raise ValueError("the stream is on %s, the tensors are on %s" % (stream.device, x.device))
        with torch.cuda.stream(stream):
            return call()
    if x.get_device() != torch._C._cuda_getDevice():
        with torch.cuda.device(x.device):
            return call()
    return call()


def _row_pitch(x: torch.Tensor, name: str) -> int:
    """Elements between neighbouring rows (vectors along the last dimension)."""
    c = x.shape[-1]
    if x.is_contiguous():
        return c
    sizes = [(n, s) for n, s in zip(x.shape[:-1], x.stride()[:-1]) if n != 1]
    pitch = sizes[-1][1] if sizes else c
    for (_, outer), (n, inner) in zip(sizes, sizes[1:]):
        if outer != n * inner:
            raise ValueError("%s: its rows are not at one pitch" % name)
    if pitch < c or (c > 1 and x.stride(-1) != 1):
        raise ValueError("%s: its rows must be dense and apart" % name)
    return pitch


def layer_norm(x: torch.Tensor, gamma: Optional[torch.Tensor] = None,
               beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
               out: Optional[torch.Tensor] = None, save: bool = False, stream=None):
    """Layer norm of x [..., c] over its last dimension; gamma, beta: float32 [c].
    With ``save`` also what ``layer_norm_backward`` needs."""
    c = x.shape[-1]
    dtype = _dtype_of(x, "x")
    for t, name in ((gamma, "gamma"), (beta, "beta")):
        _need(t, name, x, (c,), torch.float32)
    _need(out, "out", x, x.shape, x.dtype)
    _no_graph(x, gamma, beta)

    def call():
        y = x.new_empty(x.shape) if out is None else out
        rows = x.numel() // c if c else 0
        mean = rstd = None
        if save:
            mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind()
        d = rt3d.make_norm_desc(rows, c, dtype, eps, _row_pitch(x, "x"), _row_pitch(y, "out"))
        rt3d.rt3d_layernorm_fwd(d, x, gamma, beta, y, mean, rstd)
        return (y, (mean, rstd)) if save else y

    return _launch(x, stream, call)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, gamma: Optional[torch.Tensor], saved,
                        stream=None):
    """(dx, dgamma, dbeta) of ``layer_norm(x, gamma, ..., save=True)``; dx has x's
    layout."""
    c = x.shape[-1]
    dtype = _dtype_of(x, "x")
    rows = x.numel() // c if c else 0
    mean, rstd = saved
    _need(dy, "dy", x, x.shape, x.dtype)
    _need(gamma, "gamma", x, (c,), torch.float32)
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        _need(t, name, x, (rows,), torch.float32)

    def call():
        d = rt3d.make_norm_desc(rows, c, dtype, 1.0, _row_pitch(x, "x"), _row_pitch(dy, "dy"))
        dx = x.new_empty_strided(x.shape, x.stride())
        dgamma, dbeta = x.new_empty((2, c), dtype=torch.float32).unbind()
        ws = x.new_empty(rt3d.rt3d_layernorm_bwd_workspace_size(d) // 4, dtype=torch.float32)
        rt3d.rt3d_layernorm_bwd(d, x, dy, gamma, mean, rstd, dx, dgamma, dbeta, ws)
        return dx, dgamma, dbeta

    return _launch(x, stream, call)


def _rows_of(x: torch.Tensor, width: int, name: str):
    """(pitch, batch) of a [n, tokens, ...] tensor whose tokens hold ``width``
    dense elements; None where it is tight."""
    if x.is_contiguous():
        return None
    sizes, steps = x.shape, x.stride()
    inner = 1
    for i in range(len(sizes) - 1, 1, -1):
        size = sizes[i]
        if size != 1 and steps[i] != inner:
            raise ValueError("%s: a token's vectors must be dense" % name)
        inner *= size
    pitch = steps[1] if sizes[1] > 1 else width
    if pitch < width or (sizes[0] > 1 and steps[0] <= 0 and x.numel()):
        raise ValueError("%s: its tokens or clips share memory" % name)
    return pitch, steps[0] if sizes[0] > 1 else 0


def rope3d(x: torch.Tensor, grid: Sequence[int], sections: Sequence[int], base: float = 10000.0,
           t0: int = 0, pos: Optional[torch.Tensor] = None, halves: bool = False,
           inverse: bool = False, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Rotates the vectors of x [n, tokens, vecs, d] by their token's place in the
    (t, h, w) ``grid``, or by ``pos`` (int32 [n, tokens, 3]).  ``sections``: the
    channels that turn with time, row and column.  ``inverse`` turns back: the
    backward pass.  ``out`` may be x."""
    n, tokens, vecs, d = x.shape
    dtype = _dtype_of(x, "x")
    if len(grid) != 3 or len(sections) != 3:
        raise ValueError("grid and sections have three axes")
    if grid[0] * grid[1] * grid[2] != tokens:
        raise ValueError("a %s grid has not %d tokens" % (tuple(grid), tokens))
    _need(out, "out", x, x.shape, x.dtype)
    _need(pos, "pos", x, (n, tokens, 3), torch.int32)
    _no_graph(x)

    def call():
        y = x.new_empty(x.shape) if out is None else out
        desc = rt3d.make_rope_desc(n, grid, vecs, d, sections, dtype, base, t0, halves, inverse,
                                   _rows_of(x, vecs * d, "x"), _rows_of(y, vecs * d, "out"))
        rt3d.rt3d_rope3d(desc, x, pos, y)
        return y

    return _launch(x, stream, call)


def _diffattn_desc(q, k, v, lam, q_len, k_len, frame, scale, o=None, d_o=None):
    """Checks the tensors of differential attention and fills its descriptor."""
    if q.dim() != 5 or q.shape[3] != 2:
        raise ValueError("q must be [n, lq, hq, 2, d], not %s" % list(q.shape))
    n, lq, hq, _, d = q.shape
    if k.dim() != 5:
        raise ValueError("k must be [n, lk, hk, 2, d], not %s" % list(k.shape))
    lk, hk = k.shape[1:3]
    _need(k, "k", q, (n, lk, hk, 2, d), q.dtype)
    _need(v, "v", q, (n, lk, hk, 2 * d), q.dtype)
    _need(lam, "lam", q, (hq,), torch.float32)
    _need(q_len, "q_len", q, (n,), torch.int32)
    _need(k_len, "k_len", q, (n,), torch.int32)
    _need(o, "out", q, (n, lq, hq, 2 * d), q.dtype)
    _need(d_o, "do", q, (n, lq, hq, 2 * d), q.dtype)
    if scale is not None and not 0 < ctypes.c_float(scale).value < float("inf"):
        raise ValueError("scale must be > 0 and finite in 32 bits (None: 1 / sqrt(d)), got %s" % scale)
    row_q, row_k = hq * 2 * d, hk * 2 * d
    return rt3d.make_diffattn_desc(n, lq, lk, hq, hk, d, _dtype_of(q, "q"), frame, scale or 0.0,
                                   q=_rows_of(q, row_q, "q"), k=_rows_of(k, row_k, "k"),
                                   v=_rows_of(v, row_k, "v"),
                                   o=None if o is None else _rows_of(o, row_q, "out"),
                                   d_o=None if d_o is None else _rows_of(d_o, row_q, "do"))


def diff_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor,
                   frame: int = 0, q_len: Optional[torch.Tensor] = None,
                   k_len: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                   out: Optional[torch.Tensor] = None, save: bool = False, stream=None):
    """Differential attention: q [n, lq, hq, 2, d], k [n, lk, hk, 2, d], v [n, lk,
    hk, 2 d], lam float32 [hq] -> [n, lq, hq, 2 d].  ``frame`` tokens make a frame of
    the causal mask (0: none); ``q_len``, ``k_len`` (int32 [n]): the clips' lengths in
    a padded batch or a cache; what lies behind them may be anything, but what only
    the frames' mask hides must be finite.  With ``save`` also what
    ``diff_attention_backward`` needs."""
    desc = _diffattn_desc(q, k, v, lam, q_len, k_len, frame, scale, o=out)
    _no_graph(q, k, v, lam)
    n, lq, hq, _, d = q.shape
    shape = (n, lq, hq, 2 * d)

    def call():
        o = q.new_empty(shape) if out is None else out
        o2 = lse = ws = None
        if save:
            o2 = q.new_empty(shape)
            lse = q.new_empty((2, n, hq, lq), dtype=torch.float32)
        nbytes = rt3d.rt3d_diffattn_fwd_workspace_size(desc)
        if nbytes:
            ws = q.new_empty(nbytes // 4, dtype=torch.float32)
        rt3d.rt3d_diffattn_fwd(desc, q, k, v, lam, q_len, k_len, o, o2, lse, ws)
        return (o, (o, o2, lse)) if save else o

    return _launch(q, stream, call)


def diff_attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                            lam: torch.Tensor, saved, frame: int = 0,
                            q_len: Optional[torch.Tensor] = None,
                            k_len: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                            stream=None):
    """(dq, dk, dv, dlam) of ``diff_attention(..., save=True)`` with the same
    arguments."""
    o, o2, lse = saved
    desc = _diffattn_desc(q, k, v, lam, q_len, k_len, frame, scale, o=o, d_o=do)
    n, lq, hq = q.shape[:3]
    _need(o2, "o2", q, do.shape, q.dtype)
    _need(lse, "lse", q, (2, n, hq, lq), torch.float32)

    def call():
        dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
        dlam = lam.new_empty(hq)
        nbytes = rt3d.rt3d_diffattn_bwd_workspace_size(desc)
        ws = q.new_empty(nbytes // 4, dtype=torch.float32) if nbytes else None
        rt3d.rt3d_diffattn_bwd(desc, q, k, v, lam, q_len, k_len, o, o2, lse, do, dq, dk, dv, dlam, ws)
        return dq, dk, dv, dlam

    return _launch(q, stream, call)
