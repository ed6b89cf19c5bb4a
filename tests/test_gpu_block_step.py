"""Residual norm and gated feed-forward as a block uses them: around the group attention, captured, on other streams, two at once."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import gated_ffn, moga_attention, residual_norm

from . import block_parts_ref as ref
from .block_ref import near

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


# ---- one block: norm and modulation, router and attention, gated residual and norm, feed-forward, gated residual ----
N, H, D, M, F, EACH = 600, 2, 64, 3, 152, 250
C = H * D


def _params():
    p = dict(wq=_rnd(1, C, 3 * C) * C ** -0.5, wo=_rnd(2, C, C) * C ** -0.5, router=_rnd(3, M, C), w_in=_rnd(4, 2 * F, C) * C ** -0.5,
             w_out=_rnd(5, C, F) * F ** -0.5, norm=_rnd(6, C) * 0.2 + 1, post=_rnd(7, C) * 0.2 + 1)
    for i, k in enumerate(("gate1", "scale1", "shift1", "gate2", "scale2", "shift2")):
        p[k] = _rnd(10 + i, 3, C) * 0.4
    return p


def _block(x, p):
    kw = dict(tokens_per_row=EACH, eps=1e-5)
    _, h = residual_norm(x, scale=p["scale1"], shift=p["shift1"], weight=p["norm"], pre="layer", **kw)
    q, k, v = (t.contiguous().view(N, H, D) for t in (h @ p["wq"]).chunk(3, -1))
    o, _, group = moga_attention(h.detach(), p["router"], q, k, v, D ** -0.5)
    r, h = residual_norm(x, o.view(N, C) @ p["wo"], gate=p["gate1"], post_weight=p["post"], post="rms", scale=p["scale2"], shift=p["shift2"], pre="rms",
                         residual_scale=0.7, **kw)
    y = gated_ffn(h, p["w_in"], p["w_out"], "gelu_tanh")
    out, none = residual_norm(r, y, gate=p["gate2"], pre="none", **kw)
    assert none is None
    return out, group


def _block64(x, p, group):
    """The same in 64 bits with torch's own operators; the assignment is the kernels'."""
    row = torch.arange(N, device=x.device) // EACH
    ln = lambda t: (t - t.mean(1, keepdim=True)) * ((t - t.mean(1, keepdim=True)).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    rms = lambda t: t * (t.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    h = ln(x) * p["norm"] * (1 + p["scale1"][row]) + p["shift1"][row]
    q, k, v = (t.reshape(N, H, D).transpose(0, 1) for t in (h @ p["wq"]).chunk(3, -1))
    same = group[:, None] == group[None]
    s = (q @ k.transpose(1, 2) * D ** -0.5).masked_fill(~same, float("-inf"))
    gate = torch.softmax(h.detach() @ p["router"].T, -1).gather(1, group.long()[:, None])
    o = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(N, C) * gate
    t = o @ p["wo"]
    r = x + 0.7 * p["gate1"][row] * (rms(t) * p["post"])
    h = rms(r) * (1 + p["scale2"][row]) + p["shift2"][row]
    a, u = (h @ p["w_in"].T).chunk(2, -1)
    y = (ref.activation(a, "gelu_tanh")[0] * u) @ p["w_out"].T
    return r + p["gate2"][row] * y, 1e-5 / (t.square().mean(1) + 1e-5)


def test_a_block_and_its_gradients():
    """fp32 calls against 64 bits.  Some ten sums of up to 600 values and 2^-24 each behind each other: 1e-5 of a result's size is room for 16 u
    of relative error a step.  The router's gradient goes through its probability g, which multiplies a token's whole attention output, and then through the
    RMS norm of t = g w: norm(g w) depends on g by eps alone.  With n = t / sqrt(m + eps), m = mean t^2, and e the gradient of n, dL/dg = sum_c e_c dn_c/dg =
    sum_c e_c n_c / g (1 - m / (m + eps)) = sum_c e_c n_c / g eps / (m + eps), the difference of two terms 1 / (eps / (m + eps)) times its size, each
    with 1e-5 of itself."""
    x, p, d = _rnd(30, N, C).requires_grad_(), {k: v.requires_grad_() for k, v in _params().items()}, _rnd(31, N, C)
    out, group = _block(x, p)
    grads = torch.autograd.grad(out, [x, *p.values()], d)
    x64, p64 = x.detach().double().requires_grad_(), {k: v.detach().double().requires_grad_() for k, v in p.items()}
    out64, left = _block64(x64, p64, group)
    near(out, out64, 1e-5, "out")
    for k, g, w in zip(["x", *p], grads, torch.autograd.grad(out64, [x64, *p64.values()], d.double())):
        near(g, w, 1e-5 / float(left.detach().min()) if k == "router" else 1e-5, k)


# ---- the calls as such ----
def _calls(dtype=BF, n=900, c=264, f=520):
    t = {k: _rnd(i, n, c).to(dtype) for i, k in enumerate(("x", "y", "d_r", "d_h"))}
    rows = {k: _rnd(20 + i, 3, c) for i, k in enumerate(("gate", "scale", "shift"))}
    one = {k: _rnd(25 + i, c) for i, k in enumerate(("post_weight", "weight", "bias"))}
    wi, wo = (_rnd(40, 2 * f, c) * c ** -0.5).to(dtype), (_rnd(41, c, f) * f ** -0.5).to(dtype)
    few, how = t["x"][:5].contiguous(), dict(y=t["y"], **rows, **one, post="rms", pre="layer", tokens_per_row=400)

    def run(**kw):
        r, h, stats = mg.moga_residual_norm_fwd(t["x"], **how, **kw)
        d = mg.moga_residual_norm_bwd(t["d_r"], t["d_h"], t["x"], stats, **how, **kw)
        y, au, hh = mg.moga_gated_ffn_fwd(h, wi, wo, **kw)
        g = mg.moga_gated_ffn_bwd(t["d_r"], h, wi, wo, au, hh, **kw)
        one = mg.moga_gated_ffn_fwd(few, wi, wo, want_saved=False, **kw)[0]
        return [r, h, stats, *d, y, au.view(torch.uint8), hh, *g, one]   # bits behind [a, u] are no numbers
    return run


@pytest.mark.parametrize("dtype", [BF, F32])
def test_graph(dtype):
    """Captured and replayed with eager work between, and two graphs whose temporaries come from the same pool."""
    run = _calls(dtype)
    eager = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    a, b = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(a):
        first = run()
    with torch.cuda.graph(b, pool=a.pool()):
        second = run()
    for _ in range(3):
        for t in (*first, *second):
            t.fill_(7)
        for g, got in ((a, first), (b, second)):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, eager))
        again = run()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(again, eager))


def test_captured_training_step():
    """Forward and backward through autograd in one graph: the same gradients at every replay, of inputs that change between them."""
    n, c, f = 130, 136, 72
    leaves = [t.to(BF).requires_grad_() for t in (_rnd(1, n, c), _rnd(2, n, c), _rnd(3, 2 * f, c) * 0.1, _rnd(4, c, f) * 0.1)]
    gate = _rnd(5, 1, c).requires_grad_()
    d = _rnd(6, n, c).to(BF)

    def step():
        x, y, wi, wo = leaves
        r, h = residual_norm(x, y, gate=gate, post="rms", pre="layer")
        out, _ = residual_norm(r, gated_ffn(h, wi, wo), pre="none")
        return torch.autograd.grad(out, [*leaves, gate], d)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (7, 8):
        with torch.no_grad():
            leaves[0].copy_(_rnd(seed, n, c).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):   # where the leaves were first used
            want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_on_another_stream():
    run, side = _calls(), torch.cuda.Stream()
    want = run()
    torch.cuda.synchronize()
    for _ in range(3):
        got = run(stream=side)
        noise = [torch.full((900, 520), 7.0, device="cuda") for _ in range(20)]   # would take memory that is given back too early
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del noise


def test_two_calls_at_once():
    a, b = _calls(BF), _calls(F32)
    want = a(), b()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s1):
            x = a()
        with torch.cuda.stream(s2):
            y = b()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(x, want[0])) and all(torch.equal(p, q) for p, q in zip(y, want[1]))


def test_what_lies_behind_the_tensors_stays():
    """Outputs that are parts of a longer buffer are the C calls' own affair: with guards behind every tensor of the binding's calls nothing is written
    past an end (sizes that are no multiple of a tile)."""
    import ctypes
    n, c, f = 67, 72, 88
    lib, guard = mg.load(), 4096
    keep = []

    def buf(*shape, dtype=BF):
        size = torch.Size(shape).numel()
        t = torch.full((size + guard,), -7.0, device="cuda", dtype=dtype)
        keep.append((t, size))
        return t

    x, wi, wo, dy = (_rnd(i, *s).to(BF) for i, s in enumerate(((n, c), (2 * f, c), (c, f), (n, c))))
    h, au, y, dx, dwi, dwo = buf(n, f), buf(n * f * 9 // 4), buf(n, c), buf(n, c), buf(2 * f, c), buf(c, f)
    fb, bb = (max(16, mg.workspace_bytes(op, n, 0, f, 1, c, 1)) for op in (mg.OP_GATED_FFN_FWD, mg.OP_GATED_FFN_BWD))
    wf, wb = buf(-(-fb // 2)), buf(-(-bb // 2))
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.moga_gated_ffn_fwd(ptr(x), ptr(wi), ptr(wo), 1, n, c, f, 0, ptr(h), ptr(au), ptr(y), ptr(wf), fb, st) == 0
    assert lib.moga_gated_ffn_bwd(ptr(dy), ptr(x), ptr(wi), ptr(wo), ptr(au), ptr(h), 1, n, c, f, 0, ptr(dx), ptr(dwi), ptr(dwo), ptr(wb), bb, st) == 0
    torch.cuda.synchronize()
    assert all((t[size:] == -7).all() for t, size in keep)
    want = mg.moga_gated_ffn_fwd(x, wi, wo)
    assert torch.equal(y[:n * c].view(n, c), want[0]) and torch.equal(au[:n * f * 9 // 4].view(torch.uint8), want[1].view(torch.uint8))
