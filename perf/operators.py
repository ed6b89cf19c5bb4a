"""Layer norm, rotary positions and differential attention: measurable cases and their plain forms.

A case is one pass through one operator, either in its plain form (elementary torch operations in 32 bits, `own` False) or
through the entry points of `paper_2510_18692_amd` (`own` True).  Token counts, widths and group counts are those of the
attention cases: latent frames of 30 x 52 = 1,560 tokens, the 1536/12 and 5120/40 (width / heads) backbones, head_dim 128 in
bf16 and 64 or 128 in fp32.
"""
from __future__ import annotations

import math

import torch

own = False

FRAME = (30, 52)   # latent frame of 480p video, rows x columns
EPS = 1e-6
BASE = 10000.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _mg():
    from paper_2510_18692_amd import binding
    return binding


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of the hidden state before the router and the projections: latency
        dict(name="norm_one_token", op="norm", train=False, N=1, C=5120, dtype="bf16", affine=True),
        # full precision, no round size: a model's gradient checks
        dict(name="norm_f32_odd_train", op="norm", train=True, N=4099, C=1535, dtype="f32", affine=True),
        # queries (or keys) normalised per head, 21 frames of the small backbone
        dict(name="norm_heads_train", op="norm", train=True, N=32760 * 12, C=128, dtype="bf16", affine=True),
        # the hidden state of 64 frames on the large backbone
        dict(name="norm_hidden_train", op="norm", train=True, N=99840, C=5120, dtype="bf16", affine=True),
        # one new token at a far position, context stretched four times by parts: latency
        dict(name="rotary_one_token", op="rotary", train=False, N=1, H=40, D=128, R=128, axes=1, interleaved=False, scaling="parts",
             far=500000, dtype="bf16", sort=0),
        # 64 frames on the large backbone, three axes (t, y, x), neighbouring channels are a pair
        dict(name="rotary_video_train", op="rotary", train=True, N=99840, H=40, D=128, R=128, axes=3, interleaved=True, scaling=None,
             far=0, dtype="bf16", sort=0),
        # the same rotation on the way into eight groups, three quarters of the head, 21 frames of the small backbone
        dict(name="rotary_sorted_train", op="rotary", train=True, N=32760, H=12, D=128, R=96, axes=1, interleaved=False, scaling="linear",
             far=100000, dtype="bf16", sort=8),
        # one new query in each of four sequences, long lists of keys: serving
        dict(name="diff_one_query", op="diff", train=False, N=4, keys=4 * 16384, H=12, D=128, groups=4, uneven=0.5, dtype="bf16"),
        # full precision at the size that gradient checks of a model use
        dict(name="diff_f32_train", op="diff", train=True, N=4096, H=2, D=64, groups=8, uneven=0.3, dtype="f32"),
        # a short context of no round size, twenty groups of unequal length, one of them empty
        dict(name="diff_ragged_train", op="diff", train=True, N=10007, H=12, D=128, groups=20, uneven=0.8, dtype="bf16"),
        # 21 latent frames on the small backbone: one step of inference
        dict(name="diff_clip_infer", op="diff", train=False, N=32760, H=12, D=128, groups=8, uneven=0.2, dtype="bf16"),
        # 40 latent frames, eight groups
        dict(name="diff_long_train", op="diff", train=True, N=62400, H=12, D=128, groups=8, uneven=0.4, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "rotary", "diff", "diff"])
    train = rng.random() < 0.6
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice([128, 64, 512, 1536, 5120, _log(rng, 8, 8192)])
        N = _log(rng, 1, 99840 * 5120 // max(C, 512) // (2 if dtype == "f32" else 1))
        return dict(op=op, train=train, N=N, C=C, dtype=dtype, affine=rng.random() < 0.8)
    if op == "rotary":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        D = 128 if dtype == "bf16" else rng.choice([64, 128])
        H = rng.choice([2, 3, 12, 12, 40])
        N = _log(rng, 1, 99840 * 40 // H // (2 if dtype == "f32" else 1) // (1 if H == 40 else 2))
        axes = rng.choice([1, 1, 3])
        R = rng.choice([D, D, D // 2, D // 4 * 3, D - 4])
        return dict(op=op, train=train, N=N, H=H, D=D, R=R, axes=axes, interleaved=rng.random() < 0.5,
                    scaling=rng.choice([None, "linear", "base", "parts"]), far=rng.choice([0, 5000, 300000, 1000000]), dtype=dtype,
                    sort=rng.choice([0, 1, 5, 16]))
    if not train and rng.random() < 0.4:   # a few queries a group
        groups = rng.randint(1, 8)
        return dict(op=op, train=False, N=groups * rng.choice([1, 1, 1, 2, 7]), keys=groups * _log(rng, 16, 40000), H=rng.choice([3, 12, 40]), D=128,
                    groups=groups, uneven=rng.uniform(0, 0.8), dtype="bf16")
    if rng.random() < 0.25:
        return dict(op=op, train=train, N=_log(rng, 16, 6000), H=rng.randint(1, 4), D=rng.choice([64, 128]), groups=rng.choice([1, 3, 8]),
                    uneven=rng.uniform(0, 0.8), dtype="f32")
    case = dict(op=op, train=train, N=_log(rng, 200, 62400), H=rng.choice([3, 4, 12, 12, 16]), D=128, groups=rng.choice([1, 4, 8, 12, 20, 40]),
                uneven=rng.uniform(0, 0.8), dtype="bf16")
    most = max(work(c)["flops"] for c in listed())
    while work(case)["flops"] > 0.8 * most:
        case["N"] //= 2
    return case


def _sizes(total, groups, uneven):
    """Lengths that sum to `total`: geometric, the last one empty where they differ much and there are many."""
    ratio = 1 - uneven / max(2, groups / 2)
    w = [ratio ** i for i in range(groups)]
    if uneven > 0.6 and groups >= 12:
        w[-1] = 0.0
    cut, at = [0], 0.0
    for x in w:
        at += x / sum(w)
        cut.append(min(total, int(round(at * total))))
    cut[-1] = total
    if w[-1] == 0.0:
        cut[-2] = total
    return cut


def _bounds(case):
    if "keys" in case:   # as many queries in every group, lists of keys of unequal length
        n = case["N"] // case["groups"]
        return [n * g for g in range(case["groups"] + 1)], _sizes(case["keys"], case["groups"], case["uneven"])
    cut = _sizes(case["N"], case["groups"], case["uneven"])
    return cut, cut


def work(case):
    """Every input read once and every output written once; the operations of the formulas."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        e = case["N"] * case["C"]
        return {"bytes": (4 if case["train"] else 2) * e * es + 16 * case["C"], "flops": (22 if case["train"] else 8) * e}
    if case["op"] == "rotary":
        e = case["N"] * case["H"] * case["D"]
        passes = (2 if case["train"] else 1) * (3 if case["sort"] else 2)
        return {"bytes": 2 * passes * e * es, "flops": 4 * passes * e}
    cq, ck = _bounds(case)
    pairs = case["H"] * sum((cq[g + 1] - cq[g]) * (ck[g + 1] - ck[g]) for g in range(case["groups"]))
    rows = case["H"] * case["D"] * es
    fwd = rows * (2 * cq[-1] + 2 * ck[-1])
    bwd = rows * (2 * cq[-1] + 2 * ck[-1]) if case["train"] else 0
    return {"bytes": fwd + bwd, "flops": pairs * case["D"] * (16 if case["train"] else 6)}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _axis_pairs(R, axes):
    """Pairs of each axis: the first one gets what does not divide."""
    each = R // 2 // axes
    return [R // 2 - (axes - 1) * each] + [each] * (axes - 1)


SCALE_FACTOR, ORIGINAL_LEN, FAST, SLOW = 4.0, 32760, 32.0, 1.0


def _frequencies(case):
    """Radians per position of every pair, 64 bits, and the factor on the rotated values."""
    out = []
    for n in _axis_pairs(case["R"], case["axes"]):
        base = BASE
        if case["scaling"] == "base" and n > 1:
            base = BASE * SCALE_FACTOR ** (n / (n - 1))
        for i in range(n):
            f = base ** (-i / n)
            if case["scaling"] == "linear":
                f /= SCALE_FACTOR
            elif case["scaling"] == "parts":
                turns = ORIGINAL_LEN * f / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - SLOW) / (FAST - SLOW)))
                f = f * keep + f / SCALE_FACTOR * (1 - keep)
            out.append(f)
    return out, (0.1 * math.log(SCALE_FACTOR) + 1 if case["scaling"] == "parts" else 1.0)


def _positions(case, device):
    i = torch.arange(case["N"], device=device)
    if case["axes"] == 1:
        return (i + case["far"])[None].to(torch.int32)
    fh, fw = FRAME
    return torch.stack([i // (fh * fw) + case["far"], i // fw % fh, i % fw]).to(torch.int32)


def _randn(shape, gen, dtype, scale=1.0, shift=0.0):
    """Normal values, made in pieces of rows."""
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
    if case["op"] == "norm":
        N, C = case["N"], case["C"]
        st["x"] = _randn((N, C), gen, dt, 1.5, 0.25)
        st["w"] = _randn((C,), gen, torch.float32, 0.2, 1.0) if case["affine"] else None
        st["b"] = _randn((C,), gen, torch.float32, 0.2) if case["affine"] else None
        if case["train"]:
            st["dy"] = _randn((N, C), gen, dt)
        return st
    if case["op"] == "rotary":
        N, H, D = case["N"], case["H"], case["D"]
        sort = case["sort"] > 0
        names = ("q", "k", "v") if sort else ("q", "k")
        for n in names:
            st[n] = _randn((N, H, D), gen, dt)
        if case["train"]:
            for n in names:
                st["d" + n] = _randn((H, N, D) if sort else (N, H, D), gen, dt)
        st["pos"] = _positions(case, "cuda")
        st["pairs"] = _axis_pairs(case["R"], case["axes"])
        if own:
            st["freqs"], st["factor"] = _mg().moga_rotary_freqs(
                [2 * n for n in st["pairs"]], BASE, scaling=case["scaling"], scale_factor=SCALE_FACTOR, original_len=ORIGINAL_LEN,
                beta_fast=FAST, beta_slow=SLOW, device="cuda")
        else:
            freqs, st["factor"] = _frequencies(case)
            st["freqs"] = torch.tensor(freqs, dtype=torch.float64, device="cuda")
        if sort:   # the order that the permutation of the groups gives
            group = torch.randint(0, case["sort"], (N,), generator=gen, device="cuda")
            st["perm"] = torch.argsort(group, stable=True).to(torch.int32)
        return st
    H, D = case["H"], case["D"]
    st["bounds"] = _bounds(case)
    st["cu_q"], st["cu_k"] = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in st["bounds"])
    nq, nk = st["bounds"][0][-1], st["bounds"][1][-1]
    st["q"] = _randn((H, nq, D), gen, dt)
    st["k"] = _randn((H, nk, D), gen, dt, 1.5)
    st["v"] = _randn((H, nk, D), gen, dt)
    st["lam"] = torch.rand((H,), generator=gen, device="cuda") * 0.6 + 0.2
    st["scale"] = (D // 2) ** -0.5
    if case["train"]:
        st["do"] = _randn((H, nq, D), gen, dt)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_norm(s):
    train = s["case"]["train"]
    x = s["x"].float()
    c = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    xh = c * rstd
    y = xh if s["w"] is None else xh * s["w"] + s["b"]
    out = {"y": y.to(s["x"].dtype)}
    if train:
        dy = s["dy"].float()
        g = dy if s["w"] is None else dy * s["w"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        out["dx"] = dx.to(s["x"].dtype)
        if s["w"] is not None:
            # long sums in 64 bits, a piece of rows at a time
            dw = torch.zeros(x.shape[1], dtype=torch.float64, device=x.device)
            db = torch.zeros_like(dw)
            for a in range(0, x.shape[0], 8192):
                d = dy[a:a + 8192]
                dw += (d * xh[a:a + 8192]).sum(0, dtype=torch.float64)
                db += d.sum(0, dtype=torch.float64)
            out["dw"], out["db"] = dw.float(), db.float()
    return out


def _halves(x, R, interleaved):
    part = x[..., :R]
    return (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :R // 2], part[..., R // 2:])


def _plain_rotate(x, cos, sin, R, interleaved):
    """x [N, H, D]; cos, sin [N, 1, R / 2]; 32 bits, rounded once."""
    f = x.float()
    a, b = _halves(f, R, interleaved)
    y = f.clone()
    ya, yb = _halves(y, R, interleaved)
    ya.copy_(a * cos - b * sin)
    yb.copy_(b * cos + a * sin)
    return y.to(x.dtype)


def _plain_rotary(s):
    case = s["case"]
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(s["pairs"], device="cuda"))
    angle = s["pos"].double()[axis].t() * s["freqs"]   # far positions: 64 bits
    cos, sin = ((f(angle) * s["factor"]).float()[:, None] for f in (torch.cos, torch.sin))
    R, inter = case["R"], case["interleaved"]
    sort = case["sort"] > 0
    out = {}
    perm = s["perm"].long() if sort else None
    for n in ("q", "k"):
        y = _plain_rotate(s[n], cos, sin, R, inter)
        out[n] = y[perm].transpose(0, 1).contiguous() if sort else y
    if sort:
        out["v"] = s["v"][perm].transpose(0, 1).contiguous()
    if case["train"]:
        for n in ("q", "k", "v") if sort else ("q", "k"):
            d = s["d" + n]
            if sort:
                t = torch.empty_like(s[n])
                t[perm] = d.transpose(0, 1)
                d = t
            out["d" + n] = d if n == "v" else _plain_rotate(d, cos, -sin, R, inter)
    return out


def _head_runs(H, pairs):
    """Runs of heads whose score matrices stay under 2 GiB in 32 bits."""
    step = max(1, min(H, (1 << 29) // max(1, pairs)))
    return [(a, min(H, a + step)) for a in range(0, H, step)]


def _softmax(q, k, scale):
    p = torch.matmul(q, k.transpose(1, 2)).mul_(scale)
    p.sub_(p.amax(2, keepdim=True)).exp_()
    return p.div_(p.sum(2, keepdim=True))


def _plain_diff(s):
    case = s["case"]
    q, k, v, scale, D = s["q"], s["k"], s["v"], s["scale"], case["D"]
    train, h = case["train"], D // 2
    o = torch.zeros_like(q)
    if train:
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dlam = torch.zeros(case["H"], dtype=torch.float64, device="cuda")
    cq, ck = s["bounds"]
    for g in range(case["groups"]):
        a, b, c, d = cq[g], cq[g + 1], ck[g], ck[g + 1]
        if b == a or d == c:
            continue
        for h0, h1 in _head_runs(case["H"], (b - a) * (d - c)):
            qs, ks, vs = q[h0:h1, a:b].float(), k[h0:h1, c:d].float(), v[h0:h1, c:d].float()
            lam = s["lam"][h0:h1, None, None]
            q1, q2, k1, k2 = qs[..., :h], qs[..., h:], ks[..., :h], ks[..., h:]
            p1, p2 = _softmax(q1, k1, scale), _softmax(q2, k2, scale)
            o1, o2 = torch.matmul(p1, vs), torch.matmul(p2, vs)
            o[h0:h1, a:b] = (o1 - lam * o2).to(o.dtype)
            if not train:
                continue
            do = s["do"][h0:h1, a:b].float()
            dp = torch.matmul(do, vs.transpose(1, 2))
            d1, d2 = (do * o1).sum(2, keepdim=True), (do * o2).sum(2, keepdim=True)
            dlam[h0:h1] -= d2.sum((1, 2), dtype=torch.float64)
            dv[h0:h1, c:d] = torch.matmul((p1 - lam * p2).transpose(1, 2), do).to(dv.dtype)
            s1 = p1.mul_(dp - d1).mul_(scale)
            s2 = p2.mul_(dp.sub_(d2)).mul_(-lam * scale)
            dq[h0:h1, a:b] = torch.cat([torch.matmul(s1, k1), torch.matmul(s2, k2)], 2).to(dq.dtype)
            dk[h0:h1, c:d] = torch.cat([torch.matmul(s1.transpose(1, 2), q1), torch.matmul(s2.transpose(1, 2), q2)], 2).to(dk.dtype)
    out = {"o": o}
    if train:
        out.update(dq=dq, dk=dk, dv=dv, dlam=dlam.float())
    return out


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if not own:
        return {"norm": _plain_norm, "rotary": _plain_rotary, "diff": _plain_diff}[case["op"]](s)
    mg = _mg()
    train = case["train"]
    if case["op"] == "norm":
        y, mean, rstd = mg.moga_layer_norm_fwd(s["x"], s["w"], s["b"], EPS, want_stats=train)
        out = {"y": y}
        if train:
            out["dx"], dw, db = mg.moga_layer_norm_bwd(s["dy"], s["x"], s["w"], mean, rstd, want_dw=s["w"] is not None)
            if dw is not None:
                out["dw"], out["db"] = dw, db
        return out
    if case["op"] == "rotary":
        how = dict(axis_pairs=s["pairs"], interleaved=case["interleaved"], factor=s["factor"])
        if case["sort"]:
            out = dict(zip(("q", "k", "v"), mg.moga_rotary_permute_fwd(s["q"], s["k"], s["v"], s["perm"], s["pos"], s["freqs"], **how)))
            if train:
                d = mg.moga_rotary_permute_bwd(s["dq"], s["dk"], s["dv"], s["perm"], s["pos"], s["freqs"], **how)
                out.update(zip(("dq", "dk", "dv"), d))
            return out
        out = dict(zip(("q", "k"), mg.moga_rotary_fwd(s["q"], s["k"], s["pos"], s["freqs"], **how)))
        if train:
            out.update(zip(("dq", "dk"), mg.moga_rotary_bwd(s["dq"], s["dk"], s["pos"], s["freqs"], **how)))
        return out
    o, parts, lse = mg.moga_diff_attn_fwd(s["q"], s["k"], s["v"], s["lam"], s["cu_q"], s["cu_k"], s["scale"], want_parts=train)
    out = {"o": o}
    if train:
        dq, dk, dv, dlam = mg.moga_diff_attn_bwd(s["do"], s["q"], s["k"], s["v"], parts, lse, s["lam"], s["cu_q"], s["cu_k"], s["scale"])
        out.update(dq=dq, dk=dk, dv=dv, dlam=dlam)
    return out


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_norm(s, train):
    """Row by row definition; the gradients as products with the Jacobian of the normalised row."""
    x = s["x"].double()
    C = x.shape[1]
    mu = x.sum(1, keepdim=True) / C
    sd = torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / C + EPS)
    w = torch.ones(C, dtype=torch.float64, device="cuda") if s["w"] is None else s["w"].double()
    b = torch.zeros_like(w) if s["b"] is None else s["b"].double()
    z = (x - mu) / sd
    out = {"y": w * z + b}
    if train:
        dy = s["dy"].double()
        gz = dy * w
        out["dx"] = (gz - (gz.sum(1, keepdim=True) + z * (gz * z).sum(1, keepdim=True)) / C) / sd
        if s["w"] is not None:
            out["dw"], out["db"] = (dy * z).sum(0), dy.sum(0)
    return out


def _exact_turn(x, case, s, sign):
    """[N, H, D] as complex numbers times factor * exp(i sign angle), a piece of tokens at a time."""
    R, inter = case["R"], case["interleaved"]
    y = x.double()
    freqs, factor = _frequencies(case)
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    first = [sum(s["pairs"][:a]) for a in range(case["axes"] + 1)]
    first[-1] = R // 2
    for n0 in range(0, x.shape[0], 16384):
        angle = torch.empty((min(16384, x.shape[0] - n0), R // 2), dtype=torch.float64, device="cuda")
        for a in range(case["axes"]):
            angle[:, first[a]:first[a + 1]] = s["pos"][a, n0:n0 + 16384, None].double() * f[first[a]:first[a + 1]]
        turn = torch.polar(torch.full_like(angle, factor), sign * angle)[:, None]
        head = y[n0:n0 + 16384, :, :R]
        if inter:
            z = torch.complex(head[..., 0::2].contiguous(), head[..., 1::2].contiguous()) * turn
            head.copy_(torch.view_as_real(z).flatten(-2))
        else:
            z = torch.complex(head[..., :R // 2].contiguous(), head[..., R // 2:].contiguous()) * turn
            head.copy_(torch.cat([z.real, z.imag], -1))
    return y


def _exact_rotary(s, case):
    sort = case["sort"] > 0
    out = {}
    for n in ("q", "k", "v") if sort else ("q", "k"):
        y = s[n].double() if n == "v" else _exact_turn(s[n], case, s, 1)
        out[n] = y.index_select(0, s["perm"].long()).permute(1, 0, 2).contiguous() if sort else y
    if case["train"]:
        for n in ("q", "k", "v") if sort else ("q", "k"):
            d = s["d" + n]
            if sort:   # token t stands in slot inv[t]
                inv = torch.argsort(s["perm"].long())
                d = d.permute(1, 0, 2)[inv]
            out["d" + n] = d.double() if n == "v" else _exact_turn(d, case, s, -1)
    return out


def _exact_diff(s, case):
    """A head and a run of queries at a time, from logarithms of sums; keys' gradients added up over the runs."""
    H, D, scale = case["H"], case["D"], s["scale"]
    h = D // 2
    nq, nk = s["q"].shape[1], s["k"].shape[1]
    f64 = dict(dtype=torch.float64, device="cuda")
    o = torch.zeros((H, nq, D), **f64)
    train = case["train"]
    if train:
        dq, dk, dv, dlam = torch.zeros((H, nq, D), **f64), torch.zeros((H, nk, D), **f64), torch.zeros((H, nk, D), **f64), torch.zeros(H, **f64)
    cq, ck = s["bounds"]
    for g in range(case["groups"]):
        keys = slice(ck[g], ck[g + 1])
        if ck[g + 1] == ck[g]:
            continue
        for head in range(H):
            K, V, lam = s["k"][head, keys].double(), s["v"][head, keys].double(), float(s["lam"][head])
            step = max(1, (1 << 27) // (ck[g + 1] - ck[g]))
            for a in range(cq[g], cq[g + 1], step):
                rows = slice(a, min(cq[g + 1], a + step))
                Q = s["q"][head, rows].double()
                maps = []
                for half in (slice(0, h), slice(h, D)):
                    t = scale * (Q[:, half] @ K[:, half].T)
                    maps.append(torch.exp(t - torch.logsumexp(t, 1, keepdim=True)))
                A, B = maps
                o[head, rows] = (A - lam * B) @ V
                if train:
                    G = s["do"][head, rows].double()
                    W = G @ V.T                                # derivative by either map's weights, up to its sign and factor
                    dlam[head] -= (W * B).sum()
                    dv[head, keys] += (A - lam * B).T @ G
                    for P, half, f in ((A, slice(0, h), scale), (B, slice(h, D), -lam * scale)):
                        T = f * P * (W - (P * W).sum(1, keepdim=True))
                        dq[head, rows, half] = T @ K[:, half]
                        dk[head, keys, half] += T.T @ Q[:, half]
    out = {"o": o}
    if train:
        out.update(dq=dq, dk=dk, dv=dv, dlam=dlam)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s, case["train"])
    return _exact_rotary(s, case) if case["op"] == "rotary" else _exact_diff(s, case)
