"""Plain 64-bit statements of the block operators and bounds on the error that a 32-bit evaluation may make.

Bounds: U = 2^-23 is one rounding or truncation of a binary32 operation, BF = 2^-8 one rounding to bfloat16 (eight
significant bits: half a unit in the last place of 1.0 is 2^-8).  A sum of n products, taken in any order and with one truncation an addition, is off by
at most (n + 32) U times the sum of the products' magnitudes; the 32 covers the splitting of fp32 operands into three
bfloat16 parts (the products left out reach 2^-24 of the whole each) and the rounding of the products.  Errors of
operands propagate by |A| dB + dA |B| + dA dB.
"""
import numpy as np
import torch

U = 2.0 ** -23
BF = 2.0 ** -8
ACT_NAMES = ("silu", "gelu", "gelu_tanh", "relu")


def act64(kind, g):
    """(act(g), act'(g)) in 64 bits; kind as in the C header."""
    g = g.double()
    if kind == 0:
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    if kind == 1:
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / np.sqrt(2 * np.pi)
    if kind == 2:
        z = np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
        t = torch.tanh(z)
        return g * (1 + t) / 2, (1 + t) / 2 + g / 2 / torch.cosh(z).square() * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g * g)
    return g.clamp_min(0), (g > 0).double()


def act_err(g):
    """Absolute error of act and act' as evaluated in 32 bits with the fast exponential: its relative error grows with
    the argument as (2 + 1.2 |g|) U, and there are a handful of operations behind it; 2^-19 (1 + |g|) covers |g| <= 16."""
    return 2.0 ** -19 * (1 + g.abs())


def product(A, B, dA=0.0, dB=0.0):
    """A @ B in 64 bits and the bound on the error of its 32-bit form when A and B are off by dA and dB."""
    dA, dB = torch.zeros_like(A) + dA, torch.zeros_like(B) + dB
    mag = A.abs() @ B.abs()
    return A @ B, (A.shape[-1] + 32) * U * mag + A.abs() @ dB + dA @ B.abs() + dA @ dB


def rounded(v, dv, bf):
    """The error after one rounding to the storage type."""
    return dv + (BF if bf else U) * (v.abs() + dv)


def ffn_forward64(x, wg, wu, wd, kind, bf):
    """{name: (value, error bound)} of y, gate, up (these two before they are rounded for saving)."""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    g, dg = product(x, wg.mT)
    u, du = product(x, wu.mT)
    a, _ = act64(kind, g)
    da = 1.13 * dg + act_err(g)                   # |act'| <= 1.13 for all four
    h, dh = a * u, a.abs() * du + da * u.abs() + da * du
    y, dy = product(h, wd.mT, rounded(h, dh, bf))
    return {"y": (y, rounded(y, dy, bf)), "gate": (g, dg), "up": (u, du)}


def ffn_backward64(dy, x, wg, wu, wd, g, u, kind, bf):
    dy, x, wg, wu, wd, g, u = (t.double() for t in (dy, x, wg, wu, wd, g, u))
    dh, e = product(dy, wd)
    a, s = act64(kind, g)
    ea = act_err(g)
    dgate, eg = dh * u * s, (e * (s.abs() + ea) + dh.abs() * ea) * u.abs()
    dup, eu = dh * a, e * (a.abs() + ea) + dh.abs() * ea
    h, eh = a * u, ea * u.abs()
    eg, eu, eh = rounded(dgate, eg, bf), rounded(dup, eu, bf), rounded(h, eh, bf)
    d1, e1 = product(dgate, wg, eg)
    d2, e2 = product(dup, wu, eu)
    out = {"dx": (d1 + d2, e1 + e2 + (d1.abs() + d2.abs()) * U * (g.shape[-1] + 32))}
    out["dw_gate"] = product(dgate.mT, x, eg.mT)
    out["dw_up"] = product(dup.mT, x, eu.mT)
    out["dw_down"] = product(dy.mT, h, 0.0, eh)
    return {n: (v, rounded(v, e, bf)) for n, (v, e) in out.items()}


def within(got, value, bound, what):
    """|got - value| <= bound, element by element (NaN in both counts as equal)."""
    got = got.double()
    bad = ~((got - value).abs() <= bound) & ~(got.isnan() & value.isnan())
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst "
                                 f"{float(((got - value).abs() / (bound + 1e-300))[bad].max()):.3g} times the bound")


def act8_numpy(x):
    """(q, exponent, values) of the 8-bit form of a float32 array (rows, cols), group by group in 64 bits."""
    rows, cols = x.shape
    G = (cols + 31) // 32
    q = np.zeros((rows, cols), np.int8)
    e = np.zeros((rows, G), np.uint8)
    v = np.zeros((rows, cols), np.float64)
    for r in range(rows):
        for g in range(G):
            t = x[r, 32 * g:32 * g + 32].astype(np.float64)
            if not np.isfinite(t).all():
                e[r, g], v[r, 32 * g:32 * g + 32] = 255, np.nan
                continue
            p = -126
            while np.rint(np.abs(t).max() / 2.0 ** p) > 127:
                p += 1
            if np.rint(np.abs(t).max() / 2.0 ** p) * 2.0 ** p >= 2.0 ** 128:      # rounds past the largest binary32
                e[r, g], v[r, 32 * g:32 * g + 32] = 255, np.nan
                continue
            e[r, g] = p + 127
            q[r, 32 * g:32 * g + 32] = np.rint(t / 2.0 ** p).astype(np.int8)
            v[r, 32 * g:32 * g + 32] = np.rint(t / 2.0 ** p) * 2.0 ** p
    return q, e, v


def rotate64(x, pos, cos, sin, interleaved, back=False):
    """The first R of the last axis of x (K, M, H, D) rotated by the angles at pos (K, M); also |a| + |b| per value."""
    c, s = cos.double()[pos.long()][:, :, None], sin.double()[pos.long()][:, :, None]
    if back:
        s = -s
    R = 2 * cos.shape[1]
    i = torch.arange(R // 2, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    out, mag = x.clone(), x.abs()
    out[..., ia] = x[..., ia] * c - x[..., ib] * s
    out[..., ib] = x[..., ib] * c + x[..., ia] * s
    mag[..., ia] = mag[..., ib] = x[..., ia].abs() + x[..., ib].abs()
    return out, mag


def qk_forward64(x, w, pos, cos, sin, eps, interleaved, bf):
    """Value and bound: the sum of squares has D positive terms (D U relative, half of it in the root), then a few
    roundings more, each relative to |a| + |b|."""
    x, w = x.double(), w.double()[:, None, None]
    D = x.shape[-1]
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    v, mag = rotate64(x * r * w, pos, cos, sin, interleaved)
    return v, rounded(v, (D + 16) * U * mag, bf)


def qk_backward64(d, x, w, pos, cos, sin, eps, interleaved, bf):
    d, x, w = d.double(), x.double(), w.double()[:, None, None]
    D = x.shape[-1]
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    dn, mag = rotate64(d, pos, cos, sin, interleaved, back=True)
    xh = x * r
    m = (w * dn * xh).mean(-1, keepdim=True)
    mm = (w.abs() * mag * xh.abs()).mean(-1, keepdim=True)
    dx = r * (w * dn - xh * m)
    ex = (4 * D + 64) * U * r * (w.abs() * mag + xh.abs() * mm)
    dw = (dn * xh).sum((1, 2))
    N = x.shape[1] * x.shape[2]
    ew = (N + D + 32) * U * (mag * xh.abs()).sum((1, 2))
    return (dx, rounded(dx, ex, bf)), (dw, rounded(dw, ew, bf))
