"""Plain forms in binary64 on the CPU of the recurrent block's operators, with bounds on the error of binary32 arithmetic.

Bounds are first order in U = 2^-24 and follow the operations: every term is the largest magnitude that a rounding can apply to, times the
roundings there.  A sigmoid of g is exp2 of a rounded product (|g| U / ln 2 < 2 |g| U), the exponential, the sum and the reciprocal
(an ulp each) and a product: below (2 |g| + 8) U relative, both of f and of 1 - f.
"""
import torch

from train_util import U


def sigmoid_error(g):
    return (2 * g.abs() + 8) * U


def factors(gate, x, mode):
    """kept factor, added value, and the errors of the two (relative to a kept state, absolute)."""
    if mode == "decay":
        return gate, x, torch.zeros_like(gate), torch.zeros_like(x)
    f, i = torch.sigmoid(gate), torch.sigmoid(-gate)
    e = sigmoid_error(gate)
    # g >= 0: the kept state is h - i h, off by the error of i;  g < 0: f h
    return f, i * x, torch.where(gate >= 0, i, f) * e, i * e * x.abs()


def recurrence64(gate, x, h0, mode, lengths=None):
    """States behind every step, the last one, and bounds of both.  gate, x [T, B, n], h0 [B, n], binary64."""
    T = gate.shape[0]
    f, add, ef, ea = factors(gate, x, mode)
    # a step rounds twice, a fold of the waves before it and of the tiles before those twice more, the wave's own map twice
    h, size, err = h0, h0.abs(), torch.zeros_like(h0)
    hs, bound, before = [], [], []
    for t in range(T):
        before.append((h, err))
        size2 = f[t].abs() * size + add[t].abs()
        h2 = f[t] * h + add[t]
        err2 = f[t].abs() * err + ef[t] * size + ea[t] + 6 * U * size2
        if lengths is not None:
            here = (lengths > t)[:, None]
            h2, size2, err2 = torch.where(here, h2, h), torch.where(here, size2, size), torch.where(here, err2, err)
        h, size, err = h2, size2, err2
        hs.append(h)
        bound.append(err)
    return torch.stack(hs), torch.stack(bound), before


def recurrence_grad64(dhs, gate, x, h0, dh_last, mode, lengths=None):
    """(dgate, dx, dh0) and their bounds."""
    T = gate.shape[0]
    f, add, ef, _ = factors(gate, x, mode)
    _, _, before = recurrence64(gate, x, h0, mode, lengths)
    e, size, err = dh_last, dh_last.abs(), torch.zeros_like(dh_last)
    dg, dx, bg, bx = (torch.zeros_like(gate) for _ in range(4))
    for t in reversed(range(T)):
        total, ts = e + dhs[t], size + dhs[t].abs()
        te = err + 2 * U * ts
        h, eh = before[t]
        if mode == "blend":
            i, s = torch.sigmoid(-gate[t]), sigmoid_error(gate[t])
            slope = f[t] * i
            dx_t, bx_t = i * total, i * te + (s + 2 * U) * i * ts
            dg_t = total * (h - x[t]) * slope
            bg_t = slope * (te * (h - x[t]).abs() + ts * (eh + 2 * U * (h.abs() + x[t].abs())) + ts * (h - x[t]).abs() * (2 * s + 8 * U))
        else:
            dx_t, bx_t = total, te
            dg_t, bg_t = total * h, te * h.abs() + ts * eh + 2 * U * ts * h.abs()
        e2, size2, err2 = f[t] * total, f[t].abs() * ts, f[t].abs() * te + ef[t] * ts + 6 * U * f[t].abs() * ts
        if lengths is not None:
            here = (lengths > t)[:, None]
            zero = torch.zeros_like(e)
            dx_t, bx_t, dg_t, bg_t = (torch.where(here, v, zero) for v in (dx_t, bx_t, dg_t, bg_t))
            e2, size2, err2 = torch.where(here, e2, e), torch.where(here, size2, size), torch.where(here, err2, err)
        dg[t], dx[t], bg[t], bx[t] = dg_t, dx_t, bg_t, bx_t
        e, size, err = e2, size2, err2
    return (dg, dx, e), (bg, bx, err)


# ---- joined norms.  A row's sum has at most 96 roundings on a path (32 entries a lane, 16 waves, the butterfly and what follows).
ROUNDINGS = 96 * U


def gate64(gate, activation):
    """act(gate), its slope and the bounds of both."""
    if gate is None:
        return 1.0, 0.0, 0.0, 0.0
    if activation in (None, "none"):
        return gate, torch.ones_like(gate), 0.0, 0.0
    p, s = torch.sigmoid(gate), sigmoid_error(gate)
    if activation == "sigmoid":
        return p, p * (1 - p), p * s, p * (1 - p) * (2 * s + 2 * U)
    slope = p * (1 + gate * (1 - p))
    return gate * p, slope, gate.abs() * p * (s + 2 * U), p * (1 + gate.abs() * (1 - p)) * (2 * s + 4 * U)


def norm64(x, w, b, eps, err=0.0):
    """norm(x), mean, rstd and bounds where x is known to `err`."""
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    z = (x - mean) * rstd
    err = torch.as_tensor(err, dtype=x.dtype).expand_as(x)
    e_mean = ROUNDINGS * x.abs().mean(1, keepdim=True) + err.mean(1, keepdim=True)
    e_z = rstd * (err + e_mean + 2 * U * (x.abs() + mean.abs()))
    e_r = rstd * (ROUNDINGS + (z.abs() * e_z).mean(1, keepdim=True) + e_mean * rstd)
    y = z * w + b
    return y, (e_z + z.abs() * e_r / rstd) * w.abs() + 4 * U * (z * w).abs() + 2 * U * (b.abs() + y.abs()), mean, e_mean, rstd, e_r


def block_norm64(x, residual, w, b, gate, activation, s, w2, b2, eps):
    u, eu, mean, e_mean, rstd, e_r = norm64(x, w, b, eps)
    a, _, ea, _ = gate64(gate, activation)
    y = residual + s * a * u
    # (the scale is folded into the parameters: a rounding each)
    a_abs, ea = (a.abs(), ea) if torch.is_tensor(a) else (1.0, 0.0)
    ey = s.abs() * (a_abs * eu + ea * u.abs()) + 4 * U * (s * a * ((u - b).abs() + b.abs())).abs() + 2 * U * (y.abs() + residual.abs())
    n, en, mean_y, e_mean_y, rstd_y, e_ry = norm64(y, w2, b2, eps, ey)
    stats = torch.stack([v[:, 0] for v in (mean, rstd, mean_y, rstd_y)])
    return (y, n, stats), (ey, en, torch.stack([v[:, 0] for v in (e_mean, e_r, e_mean_y, e_ry)]))


def slope64(g, eg, z, ez, r):
    """r (g - mean g - z mean(g z)) and its bound, with g known to eg and z to ez."""
    m = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    out = r * (g - m(g) - z * m(g * z))
    size = r * (g.abs() + m(g.abs()) + z.abs() * m((g * z).abs()))
    err = r * (eg + m(eg) + z.abs() * m(eg * z.abs() + g.abs() * ez) + ez * m((g * z).abs()))
    return out, ROUNDINGS * size + err


def block_norm_grad64(dy, dn, x, y, stats, w, b, gate, activation, s, w2):
    """A dict of gradients and one of bounds.  dy or dn may be None."""
    rows = x.shape[0]
    mean, r, mean_y, ry = (v[:, None] for v in stats)
    z, ez = (x - mean) * r, 2 * U * (x.abs() + mean.abs()) * r + 2 * U * ((x - mean) * r).abs()
    G, eG = (torch.zeros_like(x), torch.zeros_like(x)) if dy is None else (dy, torch.zeros_like(dy))
    out, bound = {}, {}
    terms = ROUNDINGS + rows * U
    if dn is not None:
        zy, ezy = (y - mean_y) * ry, 2 * U * (y.abs() + mean_y.abs()) * ry + 2 * U * ((y - mean_y) * ry).abs()
        g = dn * w2
        v, ev = slope64(g, U * g.abs(), zy, ezy, ry)
        G, eG = G + v, ev + 2 * U * (G.abs() + v.abs())
        out["dnext_weight"], bound["dnext_weight"] = (dn * zy).sum(0), (dn.abs() * (ezy + terms * zy.abs())).sum(0)
        out["dnext_bias"], bound["dnext_bias"] = dn.sum(0), terms * dn.abs().sum(0)
    else:
        for key in ("dnext_weight", "dnext_bias"):
            out[key], bound[key] = torch.zeros_like(w), torch.zeros_like(w)
    a, slope, ea, es = gate64(gate, activation)
    a_abs = a.abs() if torch.is_tensor(a) else 1.0
    u = z * w + b
    eu = ez * w.abs() + 2 * U * ((z * w).abs() + b.abs())
    out["dresidual"], bound["dresidual"] = G, eG
    if gate is not None:
        out["dgate"] = G * s * u * slope
        bound["dgate"] = s.abs() * (eG * (u * slope).abs() + G.abs() * (eu * slope.abs() + u.abs() * es)) + 6 * U * out["dgate"].abs()
    g = G * s * a * w
    eg = (s * w).abs() * (eG * a_abs + G.abs() * ea) + 6 * U * g.abs()
    out["dx"], bound["dx"] = slope64(g, eg, z, ez, r)
    t = G * a
    et = eG * a_abs + G.abs() * ea + U * t.abs()
    S1, S0 = (t * z).sum(0), t.sum(0)
    e1 = (et * z.abs() + t.abs() * ez + terms * (t * z).abs()).sum(0)
    e0 = (et + terms * t.abs()).sum(0)
    out["dweight"], bound["dweight"] = s * S1, s.abs() * (e1 + 2 * U * S1.abs())
    out["dbias"], bound["dbias"] = s * S0, s.abs() * (e0 + 2 * U * S0.abs())
    out["dscale"], bound["dscale"] = w * S1 + b * S0, w.abs() * e1 + b.abs() * e0 + 4 * U * ((w * S1).abs() + (b * S0).abs())
    return out, bound
