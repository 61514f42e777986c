"""The table's, residual's and clipping operators in 64 bits on the CPU, for their tests.

Where a result is a chain of 32-bit operations, `mag` is the same chain on absolute values: every rounding on the way to a result, 2^-24 of what it
rounds, is at most that share of the magnitude, so that an error bound is a number of roundings times 2^-24 times the magnitude, and one rounding of the
result to its type."""
from types import SimpleNamespace

import numpy as np
import torch

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def embed_grad(ids, G, rows, scale):
    """(different ids ascending, their sums in float64, sums of absolute values)."""
    ids = ids.numpy().astype(np.int64)
    G = G.double().numpy()
    at = np.flatnonzero((ids >= 0) & (ids < rows))
    order = at[np.argsort(ids[at], kind="stable")]
    keys, first = np.unique(ids[order], return_index=True)
    if len(keys) == 0:
        z = np.zeros((0, G.shape[1]))
        return keys, z, z
    return keys, np.add.reduceat(G[order], first, axis=0) * scale, np.add.reduceat(np.abs(G[order]), first, axis=0) * abs(scale)


def _norm(v, mag, kind, w, b, eps):
    """hat, 1 / deviation and norm of v, and magnitudes of hat and norm."""
    if kind == "none":
        return v, torch.ones_like(v[:, :1]), v, mag, mag
    m = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1.0 / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + eps)
    hat = (v - m) * r
    hmag = (mag + (mag.mean(1, keepdim=True) if kind == "layer" else 0.0)) * r
    # the error of r: that of the mean of squares, relative to it (and to eps)
    q = (hmag * hmag).mean(1, keepdim=True)
    hmag = hmag + hat.abs() * q
    n, nmag = (hat * w, hmag * w.abs()) if w is not None else (hat, hmag)
    return (hat, r, n, hmag, nmag) if b is None else (hat, r, n + b, hmag, nmag + b.abs())


def gate(g, act):
    s = torch.sigmoid(g)
    if act == "linear":
        return g, torch.ones_like(g)
    return (s, s * (1 - s)) if act == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def residual(x, h, g, post, pre, act, pw, pb, qw, qb, eps, alpha, beta):
    """Forward, in float64, with magnitudes."""
    o = SimpleNamespace()
    y = beta * x if x is not None else torch.zeros_like(h)
    ymag = y.abs()
    if h is not None:
        o.hat, o.r, o.n, o.hat_mag, o.n_mag = _norm(h, h.abs(), post, pw, pb, eps)
        o.a, o.da = gate(g, act) if g is not None else (torch.ones(1, dtype=torch.float64), torch.zeros(1, dtype=torch.float64))
        o.a_mag = (1 + g.abs()) * o.a.abs() if g is not None else o.a     # the exponential's argument is rounded: |g| roundings more
        o.da_mag = (1 + g.abs()) * (1 + g.abs()) * torch.sigmoid(g).abs() if g is not None and act != "linear" else o.da.abs()
        y = y + alpha * o.a * o.n
        ymag = ymag + abs(alpha) * o.a_mag * o.n_mag
    o.y, o.y_mag = y, ymag
    o.y_hat, o.y_r, o.u, o.y_hat_mag, o.u_mag = _norm(y, ymag, pre, qw, qb, eps)
    return o


def _hat_grad(t, t_mag, hat, hat_mag, r, kind):
    if kind == "none":
        return t, t_mag
    rel = 1.0 + (hat_mag * hat_mag).mean(1, keepdim=True)     # the error of r
    layer = kind == "layer"
    v = r * (t - (t.mean(1, keepdim=True) if layer else 0.0) - hat * (t * hat).mean(1, keepdim=True))
    mag = r * rel * (t_mag + (t_mag.mean(1, keepdim=True) if layer else 0.0) + hat_mag * (t_mag * hat_mag).mean(1, keepdim=True))
    return v, mag


def residual_grad(x, h, g, post, pre, act, pw, pb, qw, qb, eps, alpha, beta, dy, du):
    o = residual(x, h, g, post, pre, act, pw, pb, qw, qb, eps, alpha, beta)
    z = SimpleNamespace()
    d = dy if dy is not None else torch.zeros_like(o.y)
    d_mag = d.abs()
    if du is not None:
        t = du * qw if qw is not None else du
        v, m = _hat_grad(t, t.abs(), o.y_hat, o.y_hat_mag, o.y_r, pre)
        d, d_mag = d + v, d_mag + m
        z.dpre_w = (du * o.y_hat).sum(0), (du.abs() * o.y_hat_mag).sum(0)
        z.dpre_b = du.sum(0), du.abs().sum(0)
    z.dx = beta * d, abs(beta) * d_mag
    if h is not None:
        t, t_mag = alpha * d, abs(alpha) * d_mag
        dn, dn_mag = t * o.a, t_mag * o.a_mag
        if g is not None:
            z.dg = t * o.n * o.da, t_mag * o.n_mag * o.da_mag
            z.dg_sum = z.dg[0].sum(0), z.dg[1].sum(0)
        w = pw if pw is not None else torch.ones(1, dtype=torch.float64)
        z.dh = _hat_grad(dn * w, dn_mag * w.abs(), o.hat, o.hat_mag, o.r, post)
        z.dpost_w = (dn * o.hat).sum(0), (dn_mag * o.hat_mag).sum(0)
        z.dpost_b = dn.sum(0), dn_mag.sum(0)
    return z


def check(got, want, mag, roundings, what):
    """|got - want| <= half an ulp of the result and `roundings` roundings of the magnitude."""
    got64 = got.detach().cpu().double()
    assert bool(torch.isfinite(got64).all()), f"{what}: not finite"
    tol = HALF_ULP[got.dtype] * want.abs() * (1 + 2.0 ** -7) + roundings * 2.0 ** -24 * mag + 1e-37
    worst = ((got64 - want).abs() / tol).max().item() if got64.numel() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3f} times its bound"
    return worst
