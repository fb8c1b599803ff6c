"""Plain 64-bit statements of the linear operator, the layer norm and the cross entropy, and bounds on the error that a 32-bit
evaluation may make (see _block_ref: U is one rounding of a binary32 operation or truncation, BF one to bfloat16)."""
import torch

from _block_ref import U, act64, act_err, product, rounded

NONE = 4


def act_of(kind, z):
    """act, act' and a bound on the error of either as evaluated in 32 bits."""
    if kind == NONE:
        return z, torch.ones_like(z), torch.zeros_like(z)
    return (*act64(kind, z), act_err(z))


def linear64(x, w, bias, residual, kind, bf):
    """{name: (value, error bound)} of y, and of z before it is rounded for saving."""
    z, e = product(x.double(), w.double().mT)
    if bias is not None:
        z = z + bias.double()[:, None]
        e = e + U * (z.abs() + e)
    a, _, ea = act_of(kind, z)
    y, ey = a, 1.13 * e + ea                      # |act'| <= 1.13 for all
    if residual is not None:
        y = y + residual.double()
        ey = ey + U * (y.abs() + ey)
    return {"y": (y, rounded(y, ey, bf)), "z": (z, e)}


def linear_backward64(dy, x, w, z, kind, bf):
    dy, x, w = dy.double(), x.double(), w.double()
    if kind == NONE:
        dz, e, er = dy, torch.zeros_like(dy), torch.zeros_like(dy)
    else:
        _, s, ea = act_of(kind, z.double())
        dz, e = dy * s, dy.abs() * ea + U * (dy * s).abs()
        er = rounded(dz, e, bf)                   # the products' operand; fp32: its three parts hold all of it
    out = {"dx": product(dz, w, er), "dw": product(dz.mT, x, er.mT)}
    out["db"] = dz.sum(1), (dz.shape[1] + 32) * U * dz.abs().sum(1) + e.sum(1)
    return {n: (v, rounded(v, b, bf)) for n, (v, b) in out.items()}


def norm64(x, residual, w, b, eps, bf):
    """{name: (value, bound)}: sums of D terms are off by D U of the terms' magnitudes, the rest by a few roundings each."""
    h = x.double()
    if residual is not None:
        h = h + residual.double()
    w, b, D = w.double()[:, None], b.double()[:, None], x.shape[-1]
    mean = h.mean(-1, keepdim=True)
    em = (D + 8) * U * h.abs().mean(-1, keepdim=True)
    c, ec = h - mean, em + 2 * U * (h.abs() + mean.abs())
    var = c.square().mean(-1, keepdim=True)
    ev = (D + 8) * U * var + (2 * c.abs() * ec + ec * ec).mean(-1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    er = r * (0.5 * ev / (var + eps) + 0.375 * (ev / (var + eps)).square() * 4 + 4 * U)
    y = c * r * w + b
    ey = w.abs() * (ec * (r + er) + c.abs() * er) + 4 * U * ((c * r * w).abs() + b.abs())
    return {"y": (y, rounded(y, ey, bf)), "total": (h, rounded(h, U * h.abs(), bf)), "mean": (mean[..., 0], em[..., 0]),
            "rstd": (r[..., 0], er[..., 0])}


def norm_backward64(dy, x, w, mean, rstd, dtotal, bf):
    dy, x, w, m, r = dy.double(), x.double(), w.double()[:, None], mean.double()[..., None], rstd.double()[..., None]
    M, D = x.shape[1:]
    xh, ex = (x - m) * r, 3 * U * (x.abs() + m.abs()) * r
    g = dy * w
    along = lambda t: t.mean(-1, keepdim=True)
    mg, emg = along(g), (D + 8) * U * along(g.abs())
    mx, emx = along(g * xh), (D + 8) * U * along((g * xh).abs()) + along(g.abs() * ex)
    dx = r * (g - mg - xh * mx)
    e = r * (emg + ex * (mx.abs() + emx) + xh.abs() * emx + 6 * U * (g.abs() + mg.abs() + (xh * mx).abs()))
    if dtotal is not None:
        dx = dx + dtotal.double()
        e = e + U * (dx.abs() + e)
    dw, ew = (dy * xh).sum(1), (M + 32) * U * (dy * xh).abs().sum(1) + (dy.abs() * ex).sum(1)
    db, eb = dy.sum(1), (M + 32) * U * dy.abs().sum(1)
    return {n: (v, rounded(v, b, bf)) for n, v, b in (("dx", dx, e), ("dw", dw, ew), ("db", db, eb))}


def loss64(z, t):
    """(loss, bound), (lse, bound).  e^(z - top): the argument is off by 2 U |z - top|, the exponential by 2^-21; a lane adds at
    most a thirty-second of the row's values and a few dozen partial sums follow."""
    z = z.double()
    lse = torch.logsumexp(z, -1)
    top = z.amax(-1, keepdim=True)
    far = (torch.exp(z - lse[..., None]) * torch.where(z == -float("inf"), 0.0, (z - top).abs())).sum(-1)
    e = 2 * U * far + 2.0 ** -21 + (z.shape[-1] / 32 + 64) * U
    at = z.gather(-1, t.long().clamp_min(0)[..., None])[..., 0]
    loss = torch.where(t >= 0, lse - at, 0.0)
    return (loss, torch.where(t >= 0, e + 3 * U * (lse.abs() + torch.nan_to_num(at, 0.0, 0.0, 0.0).abs() + (top[..., 0] - lse).abs()), 0.0)), (lse, e + 2 * U * (lse.abs() + top[..., 0].abs()))


def loss_backward64(d, z, t, lse, bf):
    z, lse, d = z.double(), lse.double()[..., None], torch.where(t >= 0, d, 0.0).double()[..., None]
    p = torch.exp(z - lse)
    hot = torch.zeros_like(z).scatter_(-1, t.long().clamp_min(0)[..., None], 1.0)
    v = (p - hot) * d
    rel = 3 * U * (torch.where(p > 0, z, 0.0).abs() + lse.abs()) + 2.0 ** -21
    e = d.abs() * (p * rel + 2 * U * (p + hot)) + 2.0 ** -126           # (results below the normal numbers may be flushed)
    return v, rounded(v, e, bf)
