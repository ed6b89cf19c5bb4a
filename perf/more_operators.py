"""The rest of a block around its attention: norms with gate and residual, and the gated feed-forward.  Measurable cases and their plain forms.

  residual norm   r = x + residual_scale * gate * post(y),  h = pre(r) * weight + bias, then * (1 + scale) + shift
  gated ffn       [a, u] = x W_in^T,  h = act(a) * u,  y = h W_out^T

A case is one pass through one operator, forward or forward and backward, either in its plain form (elementary torch operations in 32 bits,
`own` False) or through the entry points of `paper_2510_18692_amd` (`own` True).  Token counts and widths are those of the attention cases:
latent frames of 30 x 52 = 1,560 tokens, widths 1536 and 5120; the feed-forward is 8/3 of the width, in whole 8s or 128s.
"""
from __future__ import annotations

import math

import torch

own = False

FRAME = 1560   # tokens of a latent frame of 480p video
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _mg():
    from paper_2510_18692_amd import binding
    return binding


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token between two halves of a block, normalised before and after: latency
        dict(name="resnorm_one_token", op="norm", train=False, N=1, C=5120, stream="bf16", dtype="bf16", post="rms", pre="rms", gated=False, mod=False,
             affine=True, each=0),
        # full precision, no round size, three samples of unequal length: a model's gradient checks
        dict(name="resnorm_f32_odd_train", op="norm", train=True, N=4099, C=1535, stream="f32", dtype="f32", post="layer", pre="layer", gated=True,
             mod=True, affine=True, each=1700),
        # 21 frames of the small backbone, gate, scale and shift of each frame, the residual stream kept in 32 bits
        dict(name="resnorm_frames_train", op="norm", train=True, N=32760, C=1536, stream="f32", dtype="bf16", post="none", pre="layer", gated=True,
             mod=True, affine=False, each=FRAME),
        # 64 frames of the large backbone, one conditioning for all of them: one step of inference
        dict(name="resnorm_hidden_infer", op="norm", train=False, N=99840, C=5120, stream="bf16", dtype="bf16", post="none", pre="layer", gated=True,
             mod=True, affine=False, each=0),
        # the same tokens, norms with weights before and after, a learned gate
        dict(name="resnorm_hidden_train", op="norm", train=True, N=99840, C=5120, stream="bf16", dtype="bf16", post="rms", pre="rms", gated=True,
             mod=False, affine=True, each=0),
        # one token through the large backbone's feed-forward: its weights are read once
        dict(name="ffn_one_token", op="ffn", train=False, N=1, C=5120, F=13696, act="silu", dtype="bf16"),
        # the tokens of a small batch: serving
        dict(name="ffn_few_tokens", op="ffn", train=False, N=24, C=1536, F=4096, act="silu", dtype="bf16"),
        # full precision at the size that gradient checks of a model use
        dict(name="ffn_f32_train", op="ffn", train=True, N=2050, C=512, F=1368, act="gelu", dtype="f32"),
        # a frame and a few tokens, no round width
        dict(name="ffn_ragged_train", op="ffn", train=True, N=1563, C=1536, F=4104, act="gelu_tanh", dtype="bf16"),
        # 21 frames through the small backbone: one step of inference
        dict(name="ffn_clip_infer", op="ffn", train=False, N=32760, C=1536, F=4096, act="silu", dtype="bf16"),
        # the same in training
        dict(name="ffn_clip_train", op="ffn", train=True, N=32760, C=1536, F=4096, act="silu", dtype="bf16"),
        # 21 frames through the large backbone, in training
        dict(name="ffn_hidden_train", op="ffn", train=True, N=32760, C=5120, F=13696, act="silu", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    train = rng.random() < 0.6
    if rng.random() < 0.5:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        stream = "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice([128, 512, 1536, 5120, _log(rng, 8, 8192)])
        N = _log(rng, 1, 99840 * 5120 // max(C, 512) // (2 if stream == "f32" else 1))
        post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("rms", "rms"), ("layer", "layer"), ("rms", "layer"), ("rms", "none"), ("absent", "layer"),
                                ("absent", "rms")])
        gated, mod = post != "absent" and rng.random() < 0.7, pre != "none" and rng.random() < 0.5
        return dict(op="norm", train=train, N=N, C=C, stream=stream, dtype=dtype, post=post, pre=pre, gated=gated, mod=mod, affine=rng.random() < 0.6,
                    each=rng.choice([0, 0, FRAME, max(1, N // rng.randint(2, 30))]))
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
    if rng.random() < 0.2:
        return dict(op="ffn", train=train, N=_log(rng, 1, 6000), C=4 * _log(rng, 16, 400), F=4 * _log(rng, 32, 800), act=act, dtype="f32")
    C = rng.choice([512, 1536, 1536, 5120, 8 * _log(rng, 8, 640)])
    F = rng.choice([8 * ((8 * C // 3 + 7) // 8), 8 * _log(rng, max(8, C // 8), C // 2)])
    if not train and rng.random() < 0.6:   # a few tokens
        return dict(op="ffn", train=False, N=_log(rng, 1, 256), C=C, F=F, act=act, dtype="bf16")
    case = dict(op="ffn", train=train, N=_log(rng, 64, 99840), C=C, F=F, act=act, dtype="bf16")
    most = max(work(c)["flops"] for c in listed())
    while work(case)["flops"] > 0.5 * most:
        case["N"] //= 2
    return case


def _rows(case):
    """Rows of gate, scale and shift: token n goes by row n // each."""
    return -(-case["N"] // case["each"]) if case["each"] else 1


def work(case):
    """Every input read once and every output written once; the operations of the formulas."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        e, xs = case["N"] * case["C"], 4 if case["stream"] == "f32" else 2
        y, h = case["post"] != "absent", case["pre"] != "none"
        fwd = e * (xs + y * (es + xs) + h * es)
        bwd = e * (xs + y * es + h * es + xs * y + xs + y * es)   # reads x, y, d_h, d_r; writes d_x, d_y
        small = 4 * _rows(case) * case["C"] * (case["gated"] + 2 * case["mod"]) + 12 * case["C"]
        return {"bytes": fwd + (bwd if case["train"] else 0) + small * (2 if case["train"] else 1), "flops": e * (38 if case["train"] else 14)}
    N, C, F = case["N"], case["C"], case["F"]
    tokens, weights = N * C * es, 3 * C * F * es
    return {"bytes": (4 * tokens + 2 * weights) if case["train"] else 2 * tokens + weights, "flops": (18 if case["train"] else 6) * N * C * F}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _randn(shape, gen, dtype, scale=1.0, shift=0.0):
    """Normal values, made in pieces."""
    out = torch.empty(shape, device="cuda", dtype=dtype)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 27):
        part = flat[a:a + (1 << 27)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale).add_(shift))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    st = {"case": case}
    N, C = case["N"], case["C"]
    if case["op"] == "ffn":
        F = case["F"]
        st["x"] = _randn((N, C), gen, dt)
        st["w_in"] = _randn((2 * F, C), gen, dt, C ** -0.5)
        st["w_out"] = _randn((C, F), gen, dt, F ** -0.5)
        if case["train"]:
            st["dy"] = _randn((N, C), gen, dt)
        return st
    sd, S, f32 = TYPES[case["stream"]], _rows(case), torch.float32
    has_y, has_h = case["post"] != "absent", case["pre"] != "none"
    st["x"] = _randn((N, C), gen, sd, 1.5, 0.25)
    st["y"] = _randn((N, C), gen, dt, 1.2, -0.1) if has_y else None
    st["gate"] = _randn((S, C), gen, f32, 0.3, 0.5) if case["gated"] else None
    st["post_weight"] = _randn((C,), gen, f32, 0.2, 1.0) if case["affine"] and case["post"] in ("rms", "layer") else None
    st["weight"] = _randn((C,), gen, f32, 0.2, 1.0) if case["affine"] and has_h else None
    st["bias"] = _randn((C,), gen, f32, 0.2) if case["affine"] and case["pre"] == "layer" else None
    st["scale"] = _randn((S, C), gen, f32, 0.2) if case["mod"] else None
    st["shift"] = _randn((S, C), gen, f32, 0.2) if case["mod"] else None
    st["residual_scale"] = 0.8 if case["post"] in ("rms", "layer") else 1.0
    if case["train"]:
        st["dr"] = _randn((N, C), gen, sd) if has_y else None   # without a branch x itself goes on, and its gradient is added elsewhere
        st["dh"] = _randn((N, C), gen, dt) if has_h else None
    return st


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _expand(p, case):
    """[S, C] by token: [N, C], or [1, C] for one row."""
    return p if p.shape[0] == 1 else p[torch.arange(case["N"], device=p.device) // case["each"]]


def _sum_rows(t, case):
    """Sums over the tokens of each row, in 64 bits: [S, C] in 32."""
    each = case["each"] or case["N"]
    whole = case["N"] // each
    s = t[:whole * each].view(whole, each, -1).sum(1, dtype=torch.float64)
    if whole * each < case["N"]:
        s = torch.cat([s, t[whole * each:].sum(0, keepdim=True, dtype=torch.float64)])
    return s.float()


def _plain_stats(t, kind):
    """Normalised rows and 1 / deviation."""
    if kind == "layer":
        t = t - t.mean(1, keepdim=True)
    rstd = torch.rsqrt((t * t).mean(1, keepdim=True) + EPS)
    return t * rstd, rstd


def _plain_norm_bwd(g, th, rstd, kind):
    d = g - th * (g * th).mean(1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(1, keepdim=True)
    return d.mul_(rstd)


def _plain_norm(s):
    case = s["case"]
    pre, post = case["pre"], case["post"]
    r = s["x"].float()
    out = {}
    if s["y"] is not None:
        yh, ry = s["y"].float(), None
        if post != "none":
            yh, ry = _plain_stats(yh, post)
        z = yh if s["post_weight"] is None else yh * s["post_weight"]
        gate = None if s["gate"] is None else _expand(s["gate"], case)
        r = r + s["residual_scale"] * (z if gate is None else gate * z)
        out["r"] = r.to(s["x"].dtype)
    if pre != "none":
        rh, rr = _plain_stats(r, pre)
        h = rh if s["weight"] is None else rh * s["weight"]
        if s["bias"] is not None:
            h = h + s["bias"]
        n = h
        if case["mod"]:
            up = 1 + _expand(s["scale"], case)
            h = n * up + _expand(s["shift"], case)
        out["h"] = h.to(TYPES[case["dtype"]])
    if not case["train"]:
        return out
    d = 0.0 if s["dr"] is None else s["dr"].float()
    if pre != "none":
        dh = s["dh"].float()
        if case["mod"]:
            out["d_scale"], out["d_shift"] = _sum_rows(dh * n, case), _sum_rows(dh, case)
            dh = dh * up
        if s["weight"] is not None:
            out["d_weight"] = (dh * rh).sum(0, dtype=torch.float64).float()
            if s["bias"] is not None:
                out["d_bias"] = dh.sum(0, dtype=torch.float64).float()
            dh = dh * s["weight"]
        d = d + _plain_norm_bwd(dh, rh, rr, pre)
    out["d_x"] = d.to(s["x"].dtype)
    if s["y"] is not None:
        e = s["residual_scale"] * d
        if gate is not None:
            out["d_gate"] = _sum_rows(e * z, case)
            e = e * gate
        if s["post_weight"] is not None:
            out["d_post_weight"] = (e * yh).sum(0, dtype=torch.float64).float()
            e = e * s["post_weight"]
        out["d_y"] = (e if post == "none" else _plain_norm_bwd(e, yh, ry, post)).to(s["y"].dtype)
    return out


def _plain_act(a, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-a))
        return a * p, p * (1 + a * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(a * 0.5 ** 0.5))
        return a * p, p + a * torch.exp(-0.5 * a * a) * (2 * math.pi) ** -0.5
    k = (2 / math.pi) ** 0.5
    t = torch.tanh(k * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)


def _plain_ffn(s):
    case = s["case"]
    F, dt = case["F"], s["x"].dtype
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    au = x @ w_in.t()
    a, u = au[:, :F], au[:, F:]
    f, slope = _plain_act(a, case["act"])
    h = f * u
    out = {"y": (h @ w_out.t()).to(dt)}
    if case["train"]:
        dy = s["dy"].float()
        out["d_w_out"] = (dy.t() @ h).to(dt)
        dh = dy @ w_out
        dau = torch.cat([dh * u * slope, dh * f], 1)
        out["d_w_in"] = (dau.t() @ x).to(dt)
        out["d_x"] = (dau @ w_in).to(dt)
    return out


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _present(**values):
    return {k: v for k, v in values.items() if v is not None}


def run(s):
    case = s["case"]
    if not own:
        return _plain_ffn(s) if case["op"] == "ffn" else _plain_norm(s)
    mg = _mg()
    train = case["train"]
    if case["op"] == "ffn":
        y, au, h = mg.moga_gated_ffn_fwd(s["x"], s["w_in"], s["w_out"], activation=case["act"], want_saved=train)
        if not train:
            return {"y": y}
        d_x, d_w_in, d_w_out = mg.moga_gated_ffn_bwd(s["dy"], s["x"], s["w_in"], s["w_out"], au, h, activation=case["act"])
        return {"y": y, "d_w_out": d_w_out, "d_w_in": d_w_in, "d_x": d_x}
    how = dict(y=s["y"], gate=s["gate"], post_weight=s["post_weight"], weight=s["weight"], bias=s["bias"], scale=s["scale"], shift=s["shift"],
               post="none" if case["post"] == "absent" else case["post"], pre=case["pre"], residual_scale=s["residual_scale"],
               tokens_per_row=case["each"] or None, eps=EPS)
    r, h, stats = mg.moga_residual_norm_fwd(s["x"], want_stats=train, dtype=TYPES[case["dtype"]], **how)
    out = _present(r=r, h=h)
    if train:
        d = mg.moga_residual_norm_bwd(s["dr"], s["dh"], s["x"], stats, **how)
        for name in ("d_scale", "d_shift", "d_weight", "d_bias", "d_x", "d_gate", "d_post_weight", "d_y"):
            if getattr(d, name) is not None:
                out[name] = getattr(d, name)
    return out


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _jacobian_t(v, g, kind):
    """Of the normalised row with respect to the row v, transposed, times g."""
    C = v.shape[1]
    c = v - v.sum(1, keepdim=True) / C if kind == "layer" else v
    var = (c ** 2).sum(1, keepdim=True) / C + EPS
    t = g / var.sqrt() - c * ((g * c).sum(1, keepdim=True) / C) / var ** 1.5
    return t - t.sum(1, keepdim=True) / C if kind == "layer" else t


def _normalised(v, kind):
    c = v - v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else v
    return c / ((c ** 2).sum(1, keepdim=True) / v.shape[1] + EPS).sqrt()


def _exact_norm(s, case):
    """A run of tokens at a time, no longer than a row of the gate has; sums by row added up over the runs."""
    N, C, S, train = case["N"], case["C"], _rows(case), case["train"]
    each = case["each"] or N
    step = max(1, min(each, (1 << 24) // C))
    one = lambda p, like: torch.full((C,), like, dtype=torch.float64, device="cuda") if p is None else p.double()
    new = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")
    has_y, has_h = s["y"] is not None, case["pre"] != "none"
    w, b, wp, alpha = one(s["weight"], 1.0), one(s["bias"], 0.0), one(s["post_weight"], 1.0), s["residual_scale"]
    r_all, h_all, dx, dy = (new(N, C) if on else None for on in (has_y, has_h, train, train and has_y))
    ds, dsh, dg, dw, db, dwp = new(S, C), new(S, C), new(S, C), new(C), new(C), new(C)
    for row in range(S):
        up = 1 + one(s["scale"][row] if case["mod"] else None, 0.0)
        down = one(s["shift"][row] if case["mod"] else None, 0.0)
        gate = one(s["gate"][row] if case["gated"] else None, 1.0)
        for a in range(row * each, min(N, (row + 1) * each), step):
            part = slice(a, min(N, (row + 1) * each, a + step))
            r = s["x"][part].double()
            if has_y:
                y = s["y"][part].double()
                yn = y if case["post"] == "none" else _normalised(y, case["post"])
                r = r + alpha * gate * (wp * yn)
                r_all[part] = r
            if has_h:
                rn = _normalised(r, case["pre"])
                h_all[part] = (w * rn + b) * up + down
            if not train:
                continue
            d = new(*r.shape) if s["dr"] is None else s["dr"][part].double()
            if has_h:
                dh = s["dh"][part].double()
                ds[row] += (dh * (w * rn + b)).sum(0)
                dsh[row] += dh.sum(0)
                dw += (dh * up * rn).sum(0)
                db += (dh * up).sum(0)
                d = d + _jacobian_t(r, dh * up * w, case["pre"])
            dx[part] = d
            if has_y:
                dg[row] += alpha * (d * wp * yn).sum(0)
                dwp += alpha * (d * gate * yn).sum(0)
                e = alpha * gate * wp * d
                dy[part] = e if case["post"] == "none" else _jacobian_t(y, e, case["post"])
    out = _present(r=r_all, h=h_all)
    if train:
        if case["mod"]:
            out.update(d_scale=ds, d_shift=dsh)
        if s["weight"] is not None:
            out["d_weight"] = dw
        if s["bias"] is not None:
            out["d_bias"] = db
        out["d_x"] = dx
        if case["gated"]:
            out["d_gate"] = dg
        if s["post_weight"] is not None:
            out["d_post_weight"] = dwp
        if has_y:
            out["d_y"] = dy
    return out


def _exact_act(a, act):
    if act == "silu":
        e = torch.exp(-a.abs())
        sig = torch.where(a >= 0, 1 / (1 + e), e / (1 + e))
        return a * sig, sig + a * sig * (1 - sig)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-a / math.sqrt(2))
        return a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    c0 = math.sqrt(2 / math.pi)
    v = c0 * (a + 0.044715 * a ** 3)
    sech2 = 1 / torch.cosh(v) ** 2
    return a / 2 * (1 + torch.tanh(v)), (1 + torch.tanh(v)) / 2 + a / 2 * sech2 * c0 * (1 + 0.134145 * a ** 2)


def _exact_ffn(s, case):
    """A run of tokens at a time; the weights' gradients added up over the runs."""
    N, F, train = case["N"], case["F"], case["train"]
    gate, up = s["w_in"][:F].double(), s["w_in"][F:].double()
    out_w = s["w_out"].double()
    y, dx = torch.empty((N, case["C"]), dtype=torch.float64, device="cuda"), None
    if train:
        dx, d_gate, d_up, d_out = torch.empty_like(y), torch.zeros_like(gate), torch.zeros_like(up), torch.zeros_like(out_w)
    for n in range(0, N, 4096):
        x = s["x"][n:n + 4096].double()
        a, u = x.mm(gate.T), x.mm(up.T)
        f, slope = _exact_act(a, case["act"])
        y[n:n + 4096] = (f * u).mm(out_w.T)
        if train:
            g = s["dy"][n:n + 4096].double()
            d_out.addmm_(g.T, f * u)
            dh = g.mm(out_w)
            da, du = dh * u * slope, dh * f
            d_gate.addmm_(da.T, x)
            d_up.addmm_(du.T, x)
            dx[n:n + 4096] = da.mm(gate) + du.mm(up)
    if not train:
        return {"y": y}
    return {"y": y, "d_w_out": d_out, "d_w_in": torch.cat([d_gate, d_up]), "d_x": dx}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_ffn(s, case) if case["op"] == "ffn" else _exact_norm(s, case)
