"""Plain 64-bit references of the token operators (CPU), and the error bounds
their GPU tests assert.  u = 2^-24 is half a step of float32, h half a step of the
layer's type (relative); a sum of K float32 terms in any order is off by at most
K u sum |terms|, and the kernels' sums run at most ``depth`` terms deep."""
import math

import torch

U = 2.0 ** -24
TDT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {k: torch.finfo(v).eps / 2 for k, v in TDT.items()}
# half of the smallest number's step: what rounding may cost near zero
TINY = {"f32": 0.0, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def rounded(x, dtype):
    """(tensor in the type, the same values in 64 bits)."""
    t = x.to(TDT[dtype])
    return t, t.double()


def within(got, ref, bound, label):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (label, got.shape, ref.shape)
    assert bool(torch.isfinite(got).all()), label
    err = (got - ref).abs()
    ratio = torch.where(err > 0, err / bound.clamp_min(1e-300), torch.zeros_like(err))
    worst = ratio.max().item() if ratio.numel() else 0.0
    print(f"{label}: worst |err|/bound {worst:.3f}", flush=True)
    assert worst <= 1.0, (label, worst)


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------

def layer_norm(x, gamma, beta, eps):
    """(y, h, mean, rstd) of rows x [rows, c]."""
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * rstd
    return h * gamma + beta, h, mean, rstd


def layer_norm_grads(dy, h, rstd, gamma):
    g = dy * gamma
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def norm_depth(c):
    """Longest chain of float32 additions in a sum over a row: a lane's share and
    the tree over lanes (the long form: c / 256 and the tree)."""
    return c // 64 + 48


def norm_h_error(x, h, rstd, c):
    """|h - h computed|: the mean is off by depth u mean|x|, the variance by twice
    depth u relatively and by the mean's error squared, rstd by half of that and
    three roundings; subtracting and scaling round twice more."""
    k = norm_depth(c)
    mean = (k + 2) * U * x.abs().mean(1, keepdim=True) * rstd
    return mean + (h.abs() + mean) * ((k + 8) * U + mean ** 2) + 2 * U * x.abs() * rstd


# ---------------------------------------------------------------------------
# Rotation by positions
# ---------------------------------------------------------------------------

def rope(x, pos, sections, base, halves, inverse):
    """x [n, tokens, vecs, d], pos [n or 1, tokens, 3]: every pair turned by hand."""
    y = x.clone()
    at = 0
    for axis, size in enumerate(sections):
        for i in range(size // 2):
            a, b = (at + i, at + i + size // 2) if halves else (at + 2 * i, at + 2 * i + 1)
            th = pos[..., axis].double() * base ** (-2.0 * i / size)
            if inverse:
                th = -th
            c, s = torch.cos(th)[..., None], torch.sin(th)[..., None]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
        at += size
    return y


def grid_positions(t, h, w, t0=0):
    g = torch.meshgrid(torch.arange(t0, t0 + t), torch.arange(h), torch.arange(w), indexing="ij")
    return torch.stack(g, -1).reshape(1, -1, 3)


# ---------------------------------------------------------------------------
# Differential attention
# ---------------------------------------------------------------------------

def visible(i, q_len, k_len, frame):
    """How many keys query i sees."""
    if not frame:
        return k_len
    p = k_len - q_len + i
    return 0 if p < 0 else min(k_len, (p // frame + 1) * frame)


def diff_attention(q, k, v, lam, frame=0, q_len=None, k_len=None, scale=None, do=None, h=0.0, tiny=0.0):
    """Everything about differential attention, query by query, from 64-bit inputs
    of the layer's values.  Returns a dict: o, o2, lse (base 2), with ``do`` also
    the gradients dq, dk, dv, dlam, and for each a bound ``*_err`` on what the
    kernels may be off, for a type whose half step is ``h`` and whose smallest
    numbers are 2 ``tiny`` apart: rounding x costs at most h |x| + tiny (below
    2^-14 an fp16 step is 2^-24 whatever the value, and probabilities over many
    keys and their gradients get there; the forward pass rounds them relative to
    the row's largest, of at least 1, so its denominator only shrinks that)."""
    n, lq, hq, _, d = q.shape
    lk, hk = k.shape[1:3]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    z = lambda *s: torch.zeros(s, dtype=torch.float64)
    r = {"o": z(n, lq, hq, 2 * d), "o2": z(n, lq, hq, 2 * d), "o_err": z(n, lq, hq, 2 * d),
         "o2_err": z(n, lq, hq, 2 * d), "lse": torch.full((2, n, hq, lq), math.inf, dtype=torch.float64)}
    for name, like in (("dq", q), ("dk", k), ("dv", v), ("dlam", lam)):
        r[name], r[name + "_err"] = torch.zeros_like(like), torch.zeros_like(like)
    for b in range(n):
        ql = lq if q_len is None else max(0, min(lq, int(q_len[b])))
        kl = lk if k_len is None else max(0, min(lk, int(k_len[b])))
        for head in range(hq):
            g, l = head // (hq // hk), float(lam[head])
            limit = torch.tensor([visible(i, ql, kl, frame) for i in range(ql)], dtype=torch.long)
            seen = torch.arange(kl)[None] < limit[:, None]
            if ql == 0 or kl == 0:
                continue
            vv = v[b, :kl, g]
            p, perr = [], []
            for m in range(2):
                qq, kk = q[b, :ql, head, m], k[b, :kl, g, m]
                s = (qq @ kk.T) * scale
                s = s.masked_fill(~seen, -math.inf)
                lse = torch.logsumexp(s, 1)
                pm = torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros(()).double())
                pm = torch.nan_to_num(pm)
                r["lse"][m, b, head, :ql] = torch.where(limit > 0, lse / math.log(2.0), math.inf)
                # A score is d products, the scaled exponent and its difference to
                # the reference round twice more (relative to the exponent's size),
                # exp2 and the sum: the relative error of a probability.
                size = (qq.abs() @ kk.abs().T) * scale
                size = torch.where(seen, size, torch.zeros(()).double())
                # the denominator's error is a mean of its terms'
                rel = U * ((d + 8) * size + 16 + (kl / 32 + 16))
                perr.append(rel + rel.max(1, keepdim=True).values)
                p.append(pm)
            mix = p[0] - l * p[1]
            weight = (p[0] * (h + perr[0]) + abs(l) * p[1] * (h + perr[1])) + tiny * (1 + abs(l)) * seen
            o, o2 = mix @ vv, p[1] @ vv
            acc = U * (kl + 8)  # accumulation over the keys
            r["o"][b, :ql, head], r["o2"][b, :ql, head] = o, o2
            both = (p[0] + abs(l) * p[1]) @ vv.abs()
            # the maps' roundings may be shared out unevenly between the two
            # products (a factor of two), and the result rounds once
            oe = 2 * weight @ vv.abs() + acc * both
            r["o_err"][b, :ql, head] = oe + h * (o.abs() + oe)
            o2e = (p[1] * (h + perr[1]) + tiny * seen) @ vv.abs() + acc * (p[1] @ vv.abs())
            r["o2_err"][b, :ql, head] = o2e + h * (o2.abs() + o2e)
            if do is None:
                continue
            g_o = do[b, :ql, head]
            dp = g_o @ vv.T
            dp_err = U * (2 * d + 2) * (g_o.abs() @ vv.abs().T)
            r["dlam"][head] -= (p[1] * dp).sum()
            r["dlam_err"][head] += (p[1] * ((perr[1] + U * (kl / 32 + 8)) * dp.abs() + dp_err)).sum()
            r["dv"][b, :kl, g] += mix.T @ g_o
            r["dv_err"][b, :kl, g] += (weight.T + U * (ql * hq + 8) * mix.abs().T) @ g_o.abs()
            for m, by in ((0, 1.0), (1, -l)):
                qq, kk = q[b, :ql, head, m], k[b, :kl, g, m]
                mean = (p[m] * dp).sum(1, keepdim=True)
                ds = by * p[m] * (dp - mean) * scale
                # the row sum comes from o and o2 as the forward pass left them
                mean_err = ((r["o_err"] + abs(l) * r["o2_err"])[b, :ql, head] if m == 0 else
                            r["o2_err"][b, :ql, head])
                mean_err = (mean_err * g_o.abs()).sum(1, keepdim=True) + \
                    U * (2 * d + 4) * ((g_o.abs() * (o.abs() + 2 * abs(l) * o2.abs())).sum(1, keepdim=True))
                lone = (limit == 1)[:, None]
                ds_err = abs(by) * scale * p[m] * ((perr[m] + h + 3 * U) * (dp - mean).abs() + (1 + h) * (dp_err + mean_err))
                ds_err = ds_err + scale * tiny * max(1.0, abs(by)) * seen
                ds, ds_err = torch.where(lone, 0.0, ds), torch.where(lone, 0.0, ds_err)
                r["dq"][b, :ql, head, m] = ds @ kk
                e = (ds_err + U * (kl + 8) * ds.abs()) @ kk.abs()
                r["dq_err"][b, :ql, head, m] = e + h * ((ds @ kk).abs() + e)
                r["dk"][b, :kl, g, m] += ds.T @ qq
                r["dk_err"][b, :kl, g, m] += (ds_err + U * (ql * hq + 8) * ds.abs()).T @ qq.abs()
    for name in ("dk", "dv"):  # one rounding of the heads' sum
        r[name + "_err"] += h * (r[name].abs() + r[name + "_err"])
    r["dlam_err"] += U * (n * lq + 8) * r["dlam_err"].abs() + U * r["dlam"].abs()
    return r
