"""Residual norm and gated feed-forward in 64 bits, from their formulas, each result with a bound on what the kernels may be off.

u = 2^-24 is half a step of fp32, `half` half a step of the outputs' type.  Sums of n values are taken as n u of the sum of their sizes; a norm's
statistics, sums of C values in pieces of at most 64 with 20 more steps, as 160 u (block_ref's layer norm)."""
import math

import torch

from .block_ref import HALF_STEP, U


def _one(p, like, x):
    return torch.full((x.shape[1],), like, dtype=torch.float64, device=x.device) if p is None else p.double()


def _stats(v, kind, eps):
    mu = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return mu, ((v - mu).square().mean(1, keepdim=True) + eps).rsqrt()


def _back(g, vh, rstd, kind):
    d = g - vh * (g * vh).mean(1, keepdim=True)
    return rstd * (d - g.mean(1, keepdim=True) if kind == "layer" else d)


def rows_of(p, N, each):
    return None if p is None else p.double()[torch.arange(N, device=p.device) // (each or max(N, 1))]


def sums_by_row(t, each):
    N = t.shape[0]
    each = each or max(N, 1)
    out = torch.zeros((max(1, -(-N // each)), t.shape[1]), dtype=torch.float64, device=t.device)
    return out.index_add_(0, torch.arange(N, device=t.device) // each, t)


def residual_norm(x, y, p, post, pre, s, each, eps, d_r=None, d_h=None, out_type=None):
    """p: gate, post_weight, weight, bias, scale, shift, each a tensor or None -> {name: (value, bound)}"""
    N, C = x.shape
    hx, hy = HALF_STEP[x.dtype], HALF_STEP[out_type or (x if y is None else y).dtype]
    X, out = x.double(), {}
    wp, w, b = _one(p["post_weight"], 1.0, x), _one(p["weight"], 1.0, x), _one(p["bias"], 0.0, x)
    gate, scale, shift = (rows_of(p[k], N, each) for k in ("gate", "scale", "shift"))
    gate = torch.ones_like(X) if gate is None else gate
    up = 1 + scale if scale is not None else torch.ones_like(X)
    shift = torch.zeros_like(X) if shift is None else shift
    r, e_r = X, torch.zeros_like(X)
    if y is not None:
        Y = y.double()
        yh, ry, e_yh = Y, torch.ones_like(Y[:, :1]), torch.zeros_like(Y)
        if post != "none":
            mu_y, ry = _stats(Y, post, eps)
            yh = (Y - mu_y) * ry
            size = Y.abs().amax(1, keepdim=True)
            e_yh = 160 * U * ry * size * (1 + ry * size)
        G = s * gate * wp
        r = X + G * yh
        e_r = G.abs() * (e_yh + 6 * U * yh.abs()) + 2 * U * (X.abs() + (G * yh).abs())
        out["r"] = (r, hx * r.abs() + e_r)
    e_rh = None
    if pre != "none":
        mu, rr = _stats(r, pre, eps)
        rh = (r - mu) * rr
        size = r.abs().amax(1, keepdim=True)
        # the norm's derivative: rstd (e - mean e - rh mean(rh e)), with mean |rh| <= 1
        e_rh = rr * (e_r + e_r.amax(1, keepdim=True) * (1 + rh.abs())) + 160 * U * rr * size * (1 + rr * size)
        W, S = w * up, b * up + shift
        h = rh * W + S
        out["h"] = (h, hy * h.abs() + W.abs() * e_rh + 6 * U * ((rh * W).abs() + (b * up).abs() + shift.abs()))
    if d_r is None and d_h is None:
        return out
    D, e_D = (torch.zeros_like(X) if d_r is None else d_r.double()), torch.zeros_like(X)

    def back(g, e_g, vh, e_vh, rstd, size, kind):
        m0, m1 = g.abs().mean(1, keepdim=True), (g * vh).abs().mean(1, keepdim=True)
        e = rstd * (e_vh * (2 * m1 + m0 * vh.abs() + m0) + 160 * U * (g.abs() + m0 + vh.abs() * m1) * (1 + (rstd * size) ** 2)
                    + (g.abs() * e_vh).mean(1, keepdim=True) * vh.abs())
        e = e + rstd * (e_g + e_g.mean(1, keepdim=True) + vh.abs() * (e_g * vh.abs()).mean(1, keepdim=True))
        return _back(g, vh, rstd, kind), e

    n_sum = N + 160
    if d_h is not None:
        dh = d_h.double()
        A1, A2 = sums_by_row(dh, each), sums_by_row(dh * rh, each)
        e1, e2 = n_sum * U * sums_by_row(dh.abs(), each), sums_by_row(dh.abs() * (e_rh + n_sum * U * rh.abs()), each)
        out["d_shift"] = (A1, e1 + U * A1.abs())
        out["d_scale"] = (w * A2 + b * A1, w.abs() * e2 + b.abs() * e1 + 4 * U * ((w * A2).abs() + (b * A1).abs()))
        out["d_weight"] = ((dh * up * rh).sum(0), (dh.abs() * up.abs() * (e_rh + (n_sum + 8) * U * rh.abs())).sum(0))
        out["d_bias"] = ((dh * up).sum(0), (n_sum + 8) * U * (dh * up).abs().sum(0))
        g = dh * W
        d, e = back(g, 4 * U * g.abs(), rh, e_rh, rr, size, pre)
        D, e_D = D + d, e + 2 * U * (D.abs() + d.abs())
    out["d_x"] = (D, hx * D.abs() + e_D)
    if y is not None:
        B, eB = sums_by_row(D * yh, each), sums_by_row(e_D * yh.abs() + D.abs() * (e_yh + (n_sum + 8) * U * yh.abs()), each)
        out["d_gate"] = (s * wp * B, (s * wp).abs() * eB + 6 * U * (s * wp * B).abs())
        out["d_post_weight"] = ((s * gate * D * yh).sum(0), (abs(s) * gate.abs() * (e_D * yh.abs() + D.abs() * (e_yh + (n_sum + 8) * U * yh.abs()))).sum(0))
        E, e_E = D * G, (e_D + 6 * U * D.abs()) * G.abs()
        d, e = (E, e_E) if post == "none" else back(E, e_E, yh, e_yh, ry, Y.abs().amax(1, keepdim=True), post)
        out["d_y"] = (d, hy * d.abs() + e)
    return out


def activation(a, kind):
    """act(a), act'(a); |act''| stays below 1.2."""
    if kind == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1 + a * (1 - p))
    if kind == "gelu":
        p = 0.5 * torch.erfc(-a / math.sqrt(2))
        return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * c * (1 + 3 * 0.044715 * a * a)


def gated_ffn(x, w_in, w_out, act, d_y=None):
    """{name: (value, bound)}.  Roundings: a, u, h, da and du once to the type, and the outputs; sums of K values to K u of their sizes; the
    activation to 8 u (2 + |a|) |a| and its derivative to 64 u (1 + |a|)^3, from an exponential whose argument is off by some |a| u (tanh's form: |a|^3)."""
    half = HALF_STEP[x.dtype]
    X, Wi, Wo = x.double(), w_in.double(), w_out.double()
    C, F = Wo.shape
    au, e_au = X @ Wi.T, C * U * (X.abs() @ Wi.abs().T)
    a, u, e_a, e_u = au[:, :F], au[:, F:], e_au[:, :F], e_au[:, F:]
    f, slope = activation(a, act)
    e_f = 8 * U * (2 + a.abs()) * a.abs() + 1.2 * e_a + 64 * U * (1 + a.abs()) ** 3 * (act == "gelu_tanh")
    h = f * u
    e_h = half * h.abs() + e_f * u.abs() + f.abs() * e_u + e_f * e_u
    y = h @ Wo.T
    out = {"y": (y, half * y.abs() + (e_h + F * U * (h.abs() + e_h)) @ Wo.abs().T), "au": (au, half * au.abs() + e_au), "h": (h, e_h)}
    if d_y is None:
        return out
    G = d_y.double()
    dh, e_dh = G @ Wo, C * U * (G.abs() @ Wo.abs())
    # from the rounded a and u
    e_a, e_u = e_a + half * a.abs(), e_u + half * u.abs()
    e_s, e_f = 1.2 * e_a + 64 * U * (1 + a.abs()) ** 3, 8 * U * (2 + a.abs()) * a.abs() + 1.2 * e_a + 64 * U * (1 + a.abs()) ** 3 * (act == "gelu_tanh")
    da, du = dh * u * slope, dh * f
    size = (dh.abs() + e_dh)
    e_da = e_dh * (u * slope).abs() + size * (e_u * (slope.abs() + e_s) + u.abs() * e_s) + half * da.abs() + 4 * U * da.abs()
    e_du = e_dh * f.abs() + size * e_f + half * du.abs() + 4 * U * du.abs()
    dau, e_dau = torch.cat([da, du], 1), torch.cat([e_da, e_du], 1)
    big = dau.abs() + e_dau
    N = X.shape[0]
    d_x, d_wi, d_wo = dau @ Wi, dau.T @ X, G.T @ h
    out["d_x"] = (d_x, half * d_x.abs() + (e_dau + 2 * F * U * big) @ Wi.abs())
    out["d_w_in"] = (d_wi, half * d_wi.abs() + (e_dau + (N + 40) * U * big).T @ X.abs())
    out["d_w_out"] = (d_wo, half * d_wo.abs() + G.abs().T @ (e_h + (N + 40) * U * (h.abs() + e_h)))
    return out
