"""Layer norm, rotary positions and differential attention in 64 bits, from their formulas, with bounds on what the kernels may be off.

u = 2^-24 is half a step of fp32; a rounding to bf16 is off by at most 2^-8 of the value.  Bounds follow the roundings that a kernel
makes: of its inputs to the matrix instructions (bf16 calls), of its output, and of fp32 sums."""
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def within(got, ref, bound, what):
    """Element by element; NaN nowhere."""
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    d = (got.double() - ref).abs()
    bad = ~(d <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {d[bad].max():.3e} at a bound of {bound.expand_as(d)[bad][d[bad].argmax()]:.3e}"


def near(got, ref, most, what):
    """Relative distance of the whole tensor."""
    den = ref.norm()
    got, ref, den = got.detach().double(), ref.detach(), den.detach()
    e = float((got - ref).norm() / den) if den > 0 else float(got.norm())
    assert e <= most, f"{what}: {e:.3e} > {most:.1e}"


def norm_fwd(x, w, b, eps):
    mu = x.mean(-1, keepdim=True)
    rstd = ((x - mu).square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = (x - mu) * rstd
    y = xh if w is None else xh * w
    return (y if b is None else y + b), mu, rstd, xh


def norm_bwd(dy, x, w, eps):
    _, _, rstd, xh = norm_fwd(x, None, None, eps)
    g = dy if w is None else dy * w
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def rotate(x, pos, freq, axis_pairs, interleaved, factor, sign=1):
    """x [N, H, D], pos [axes, N], freq [R / 2]"""
    R = 2 * freq.numel()
    axis = torch.repeat_interleave(torch.arange(pos.shape[0], device=x.device), torch.tensor(axis_pairs, device=x.device))
    a = (pos.double()[axis].t() * freq)[:, None]
    y = x.clone()
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    x1, x2 = x[..., lo], x[..., hi]
    y[..., lo] = factor * (x1 * a.cos() - sign * x2 * a.sin())
    y[..., hi] = factor * (x2 * a.cos() + sign * x1 * a.sin())
    return y


def pair_sizes(x, R, interleaved):
    """|x1| + |x2| at both places of a pair, |x| elsewhere."""
    y = x.abs()
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    s = y[..., lo] + y[..., hi]
    y = y.clone()
    y[..., lo] = s
    y[..., hi] = s
    return y


def diff_fwd(q, k, v, lam, cu_q, cu_k, scale):
    """-> o, parts [2, H, Nq, D], lse [2, H, Nq]; rows without keys: 0 and -inf"""
    H, D = q.shape[0], q.shape[2]
    h = D // 2
    parts = q.new_zeros((2, *q.shape))
    lse = q.new_full((2, *q.shape[:2]), -torch.inf)
    for g in range(len(cu_q) - 1):
        a, b, c, d = cu_q[g], cu_q[g + 1], cu_k[g], cu_k[g + 1]
        if a == b or c == d:
            continue
        for m, s in enumerate((slice(0, h), slice(h, D))):
            t = scale * q[:, a:b, s] @ k[:, c:d, s].transpose(1, 2)
            l = torch.logsumexp(t, 2)
            lse[m, :, a:b] = l
            parts[m, :, a:b] = torch.exp(t - l[..., None]) @ v[:, c:d]
    return parts[0] - lam[:, None, None] * parts[1], parts, lse


def diff_all(q, k, v, lam, do, cu_q, cu_k, scale, half):
    """Every result of a forward and a backward, and a bound for each: half = half a step of the tensors' type (matrix operands and outputs),
    fp32 for what is fp32.  -> {name: (value, bound)}"""
    H, Nq, D = q.shape
    h = D // 2
    o, parts, lse = diff_fwd(q, k, v, lam, cu_q, cu_k, scale)
    operand = half if half > U else 0.0   # weights are rounded before a bf16 product
    L = lam[:, None, None]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    e_o, e_q, e_k, e_v = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    e_parts = torch.zeros_like(parts)
    dlam, e_lam = torch.zeros_like(lam), torch.zeros_like(lam)
    worst = 0.0
    for g in range(len(cu_q) - 1):
        a, b, c, d = cu_q[g], cu_q[g + 1], cu_k[g], cu_k[g + 1]
        if a == b or c == d:
            continue
        V, dO = v[:, c:d], do[:, a:b]
        dP = dO @ V.transpose(1, 2)
        dPa = dO.abs() @ V.abs().transpose(1, 2)
        maps = []
        for m, s in enumerate((slice(0, h), slice(h, D))):
            Q, K = q[:, a:b, s], k[:, c:d, s]
            t = scale * Q @ K.transpose(1, 2)
            ta = scale * Q.abs() @ K.abs().transpose(1, 2)
            worst = max(worst, float(t.abs().max()))
            P = torch.exp(t - lse[m, :, a:b, None])
            # fp32: a score is a sum of h products (h u of their absolute sum at most, and some for scale, maximum, log-sum-exp and exp2); twice,
            # for the score and for the log-sum-exp of such scores; then sums of n weights in pieces
            rel = 2 * U * (0.5 * h * ta + 4 * t.abs() + 4 * lse[m, :, a:b, None].abs() + 64)
            maps.append((Q, K, s, P, rel.amax((1, 2), keepdim=True)))
            pv = P @ V.abs()
            e_parts[m, :, a:b] = (operand + maps[m][4]) * pv
        (_, _, _, P1, r1), (_, _, _, P2, r2) = maps
        e_o[:, a:b] = e_parts[0, :, a:b] + L.abs() * e_parts[1, :, a:b]
        A = P1 - L * P2
        Ae = r1 * P1 + L.abs() * r2 * P2 + operand * A.abs()
        dv[:, c:d] = A.transpose(1, 2) @ dO
        e_v[:, c:d] = Ae.transpose(1, 2) @ dO.abs()
        dlam -= (P2 * dP).sum((1, 2))
        e_lam += ((2 * r2 + 64 * U) * P2 * dPa).sum((1, 2))
        for m, f in ((0, torch.ones_like(L)), (1, -L)):
            Q, K, s, P, r = maps[m]
            delta = (dO * parts[m, :, a:b]).sum(2, keepdim=True)
            e_delta = (dO.abs() * e_parts[m, :, a:b]).sum(2, keepdim=True) + 64 * U * (dO.abs() * (P @ V.abs())).sum(2, keepdim=True)
            S = f * P * (dP - delta)
            Se = f.abs() * P * ((operand + r) * (dP - delta).abs() + e_delta + 64 * U * dPa)
            dq[:, a:b, s] = scale * S @ K
            e_q[:, a:b, s] = scale * Se @ K.abs()
            dk[:, c:d, s] = scale * S.transpose(1, 2) @ Q
            e_k[:, c:d, s] = scale * Se.transpose(1, 2) @ Q.abs()
    e_lse = 2 * U * (64 + 8 * worst + h * worst) * torch.ones_like(lse)
    out = {"o": (o, e_o), "dq": (dq, e_q), "dk": (dk, e_k), "dv": (dv, e_v)}
    out = {n: (r, e + half * r.abs() + 1e-30) for n, (r, e) in out.items()}
    out["parts"] = (parts, e_parts + U * parts.abs())
    out["lse"] = (lse, e_lse)
    out["dlam"] = (dlam, e_lam + U * dlam.abs())
    return out
