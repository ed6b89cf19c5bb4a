"""The residual norm, forward and backward, against 64 bits; bounds in block_parts_ref."""
import ctypes

import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import residual_norm

from . import block_parts_ref as ref
from .block_ref import within
from .test_block_parts import Args

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
PARAMS = ("gate", "post_weight", "weight", "bias", "scale", "shift")


def _inputs(N, C, stream, dtype, seed, absent=(), each=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    rows = -(-N // each) if each and N else 1
    t = dict(x=(rnd(N, C) * 1.5 + 0.25).to(stream), y=(rnd(N, C) - 0.1).to(dtype), d_r=rnd(N, C).to(stream), d_h=rnd(N, C).to(dtype))
    p = dict(gate=rnd(rows, C), post_weight=rnd(C) * 0.2 + 1, weight=rnd(C) * 0.2 + 1, bias=rnd(C), scale=rnd(rows, C) * 0.3, shift=rnd(rows, C))
    for k in absent:
        (t if k in t else p)[k] = None
    return t, p


def _run(t, p, post, pre, s, each, eps=1e-5, **kw):
    how = dict(y=t["y"], **p, post=post, pre=pre, residual_scale=s, tokens_per_row=each, eps=eps)
    r, h, stats = mg.moga_residual_norm_fwd(t["x"], dtype=None if t["y"] is not None or t["d_h"] is None else t["d_h"].dtype, **how, **kw)
    return r, h, stats, mg.moga_residual_norm_bwd(t["d_r"], t["d_h"], t["x"], stats, **how, **kw)


def _check(t, p, post, pre, s, each, eps=1e-5):
    r, h, stats, d = _run(t, p, post, pre, s, each, eps)
    want = ref.residual_norm(t["x"], t["y"], p, post, pre, s, each, eps, t["d_r"], t["d_h"], out_type=None if h is None else h.dtype)
    got = dict(d._asdict(), r=r, h=h)
    for name, value in got.items():
        given = {"d_" + k: p[k] for k in PARAMS}.get(name, True)
        if value is None:
            assert name not in want or given is None, name
        else:
            within(value, *want[name], name)
    return got


@pytest.mark.parametrize("stream,dtype", [(BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("N,C,each", [(1, 2, None), (1, 5120, None), (3, 7, 2), (37, 8, 5), (33, 63, None), (64, 128, 16), (9, 129, 1), (300, 200, 70),
                                      (41, 512, 40), (70, 513, 33), (19, 1535, 7), (50, 1536, 25), (12, 2049, None), (23, 5120, 10), (5, 8192, 2),
                                      (4, 8193, 3), (3, 16384, None)])
def test_forward_and_backward(N, C, each, stream, dtype):
    t, p = _inputs(N, C, stream, dtype, 31 * N + C, each=each)
    _check(t, p, "layer", "layer", 0.8, each)
    t, p = _inputs(N, C, stream, dtype, 31 * N + C, absent=("bias",), each=each)
    _check(t, p, "rms", "rms", -1.3, each)


@pytest.mark.parametrize("stream,dtype", [(BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("none", "rms"), ("layer", "rms"), ("rms", "layer"), ("rms", "none"), ("none", "none"),
                                      ("layer", "none"), ("absent", "layer"), ("absent", "rms")])
@pytest.mark.parametrize("C", [96, 1000, 1536])
def test_kinds(post, pre, C, stream, dtype):
    absent = ["weight", "bias", "scale", "shift", "d_h"] if pre == "none" else []
    absent += ["y", "gate", "post_weight"] if post == "absent" else ["post_weight"] if post == "none" else []
    kind = "none" if post == "absent" else post
    t, p = _inputs(130, C, stream, dtype, C, absent, each=48)
    full = _check(t, p, kind, pre, 0.7, 48)
    t, p = _inputs(130, C, stream, dtype, C, [*absent, *PARAMS])   # no parameter at all
    _check(t, p, kind, pre, 1.0, None)
    if pre != "none":
        t, p = _inputs(130, C, stream, dtype, C, [*absent, "d_r"], each=48)
        _check(t, p, kind, pre, 0.7, 48)
    assert full["d_x"].dtype == stream


@pytest.mark.parametrize("left", PARAMS)
def test_each_parameter_alone(left):
    t, p = _inputs(77, 264, F32, BF, 5, [k for k in PARAMS if k != left], each=20)
    _check(t, p, "rms", "layer", 1.0, 20)


@pytest.mark.parametrize("N,C,each", [(20011, 128, None), (20011, 128, 97), (30011, 64, 501), (20011, 250, 300), (20011, 256, None), (6000, 1536, 1560), (9001, 24, 1), (5000, 520, 2)])
def test_many_tokens_and_repeated_bits(N, C, each):
    t, p = _inputs(N, C, F32, BF, 3, each=each)
    first = _check(t, p, "rms", "layer", 1.0, each)
    for _ in range(3):
        r, h, _, d = _run(t, p, "rms", "layer", 1.0, each)
        again = dict(d._asdict(), r=r, h=h)
        assert all(torch.equal(again[k], first[k]) for k in first)


def test_against_layer_norm():
    """Alone and without modulation the norm of x is moga_layer_norm's."""
    t, p = _inputs(300, 640, BF, BF, 1, ("y", "gate", "post_weight", "scale", "shift"))
    _, h, stats = mg.moga_residual_norm_fwd(t["x"], weight=p["weight"], bias=p["bias"])
    y, mean, rstd = mg.moga_layer_norm_fwd(t["x"], p["weight"], p["bias"])
    assert (h.float() - y.float()).abs().max() <= 2.0 ** -7 * y.abs().max()   # at most a step apart
    assert torch.allclose(stats[2], mean, atol=1e-6) and torch.allclose(stats[3], rstd, rtol=1e-5)


def test_gradients_are_difference_quotients():
    """A scalar of r and h, in steps along a random direction of every input (fp32: quotients to 1e-3 of the gradient's size)."""
    t, p = _inputs(6, 40, F32, F32, 9, each=4)
    how = dict(post="layer", pre="rms", residual_scale=0.9, tokens_per_row=4, eps=1e-3)
    leaves = {k: v.clone().requires_grad_() for k, v in dict(x=t["x"], y=t["y"], **{k: p[k] for k in PARAMS if k != "bias"}).items()}
    f = lambda v: sum((o.double() * d.double()).sum() for o, d in zip(residual_norm(**v, **how), (t["d_r"], t["d_h"])))
    grads = dict(zip(leaves, torch.autograd.grad(f(leaves), list(leaves.values()))))
    for k, v in leaves.items():
        step = torch.randn_like(v)
        at = lambda h: float(f({**{n: w.detach() for n, w in leaves.items()}, k: v.detach() + h * step}))
        q, want = (at(1e-2) - at(-1e-2)) / 2e-2, float((grads[k].double() * step.double()).sum())
        assert abs(q - want) <= 2e-3 * float(grads[k].norm() * step.norm()), k


def test_bad_rows_do_not_touch_the_others():
    t, p = _inputs(40, 200, F32, F32, 9, each=10)
    r0, h0, _, d0 = _run(t, p, "rms", "layer", 1.0, 10)
    t["x"][7, 3], t["y"][25, 0], t["x"][31, 5] = float("inf"), float("nan"), -float("inf")
    r, h, _, d = _run(t, p, "rms", "layer", 1.0, 10)
    keep = [i for i in range(40) if i not in (7, 25, 31)]
    assert all(torch.equal(a[keep], b[keep]) for a, b in ((r, r0), (h, h0), (d.d_x, d0.d_x), (d.d_y, d0.d_y)))
    assert torch.equal(d.d_shift, d0.d_shift) and torch.equal(d.d_gate[1], d0.d_gate[1]) and h[25].isnan().all()


def test_constant_and_zero_rows():
    x = torch.zeros((5, 300), device="cuda")
    _, h, stats = mg.moga_residual_norm_fwd(x, pre="rms", eps=1e-4)
    assert (h == 0).all() and torch.allclose(stats[3], torch.full_like(stats[3], 100.0))
    _, h, stats = mg.moga_residual_norm_fwd(x + 3, pre="layer", eps=1e-4)
    assert (h == 0).all() and (stats[2] == 3).all()


def test_tokens_per_row_past_all_tokens():
    t, p = _inputs(50, 96, F32, BF, 8)
    want = _run(t, p, "rms", "layer", 1.0, None)
    for each in (50, 51, 2 ** 63 - 1):
        got = _run(t, p, "rms", "layer", 1.0, each)
        assert all(torch.equal(a, b) for a, b in zip((*got[:3], *got[3]), (*want[:3], *want[3])))


@pytest.mark.parametrize("N,C,each", [(1001, 5120, 1000), (1001, 520, 500), (4097, 96, 4096), (2049, 300, 1024)])
def test_short_last_row_of_the_gate_stays_in_its_workspace(N, C, each):
    t, p = _inputs(N, C, BF, BF, 11, each=each)
    _check(t, p, "rms", "rms", 1.0, each)
    _, _, stats, want = _run(t, p, "rms", "rms", 1.0, each)
    a = Args(**{k: v.data_ptr() for k, v in dict(x=t["x"], y=t["y"], **p).items()}, N=N, tokens_per_row=each, C=C, x_dtype=1, y_dtype=1, post=1, pre=1,
             residual_scale=1.0, eps=1e-5)
    need, guard = mg.workspace_bytes(mg.OP_RESIDUAL_NORM_BWD, N, 0, 0, -(-N // each), C, 1), 4 << 20
    ws = torch.full((need + guard,), 0x5a, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(v) for v in want]
    ptrs = [v.data_ptr() for v in (stats, t["d_r"], t["d_h"], *out, ws)]
    assert mg.load().moga_residual_norm_bwd(ctypes.byref(a), *map(ctypes.c_void_p, ptrs), ctypes.c_size_t(need), None) == 0
    torch.cuda.synchronize()
    assert (ws[need:] == 0x5a).all() and all(torch.equal(x, y) for x, y in zip(out, want))


def test_no_tokens():
    t, p = _inputs(0, 64, F32, BF, 1)
    r, h, _, d = _run(t, p, "rms", "layer", 1.0, 5)
    assert r.shape == h.shape == d.d_x.shape == d.d_y.shape == (0, 64)
    for k in PARAMS:
        g = getattr(d, "d_" + k)
        assert g.shape == p[k].shape and (g == 0).all()


def test_without_statistics_and_parameters():
    t, p = _inputs(90, 256, BF, BF, 4, each=30)
    how = dict(y=t["y"], **p, post="rms", pre="layer", tokens_per_row=30)
    r, h, stats = mg.moga_residual_norm_fwd(t["x"], **how)
    r2, h2, none = mg.moga_residual_norm_fwd(t["x"], want_stats=False, **how)
    assert none is None and torch.equal(r, r2) and torch.equal(h, h2)
    full = mg.moga_residual_norm_bwd(t["d_r"], t["d_h"], t["x"], stats, **how)
    some = mg.moga_residual_norm_bwd(t["d_r"], t["d_h"], t["x"], stats, want_params=False, **how)
    assert torch.equal(full.d_x, some.d_x) and torch.equal(full.d_y, some.d_y) and some[2:] == (None,) * 6


def test_autograd():
    t, p = _inputs(60, 136, F32, BF, 6, each=20)
    leaves = {k: v.clone().requires_grad_() for k, v in dict(x=t["x"], y=t["y"], **p).items()}
    how = dict(post="layer", pre="layer", residual_scale=0.5, tokens_per_row=20, eps=1e-5)
    view = lambda v: v.view(3, 20, 136)
    r, h = residual_norm(view(leaves["x"]), view(leaves["y"]), **{k: leaves[k] for k in p}, **how)
    assert r.shape == h.shape == (3, 20, 136) and r.dtype == F32 and h.dtype == BF
    torch.autograd.backward([r, h], [view(t["d_r"]), view(t["d_h"])])
    _, _, _, d = _run(t, p, "layer", "layer", 0.5, 20)
    for k, v in leaves.items():
        assert torch.equal(v.grad, getattr(d, "d_" + k)), k
    # one output used, some parameters without gradients, tensors that begin anywhere, gradients in another order
    x, w = t["x"].clone().requires_grad_(), torch.cat([p["weight"], p["weight"]]).requires_grad_()
    same, h = residual_norm(x, weight=w[1:137], shift=p["shift"], pre="rms", tokens_per_row=20, dtype=BF)
    assert same is x and h.dtype == BF
    h.backward(t["d_h"].t().contiguous().t())
    how = dict(weight=w.detach()[1:137].clone(), shift=p["shift"], pre="rms", tokens_per_row=20)
    _, _, stats = mg.moga_residual_norm_fwd(t["x"], dtype=BF, **how)
    d = mg.moga_residual_norm_bwd(None, t["d_h"], t["x"], stats, **how)
    assert torch.equal(x.grad, d.d_x) and torch.equal(w.grad[1:137], d.d_weight) and w.grad[0] == 0
    y = t["y"].clone().requires_grad_()
    r, h = residual_norm(t["x"], y, pre="layer")
    r.square().sum().backward()   # h is not used: its gradient is zeros
    # by r alone dy = 2 r, and what d_h = 0 adds is 0; one rounding of dy
    assert (y.grad.float() - 2 * r.detach()).abs().max() <= 2.0 ** -8 * (2 * r).abs().max()
    with torch.no_grad():
        again, _ = residual_norm(t["x"], y, pre="layer")
    assert torch.equal(again, r) and not again.requires_grad
    with pytest.raises(RuntimeError, match="no second derivative"):
        g, = torch.autograd.grad(residual_norm(x, pre="rms")[1].square().sum(), x, create_graph=True)
        (g.square().sum() + x.square().sum()).backward()


@pytest.mark.parametrize("post", ["none", "rms"])
def test_an_output_that_nothing_comes_of(post):
    """r alone: its gradients are those of the call without a norm of r, also where that norm divides by 0 (eps 0, r = 0); the parameters of h have zeros."""
    t, p = _inputs(12, 72, F32, F32, 2, absent=() if post == "rms" else ("post_weight",), each=5)
    t["x"][4], p["gate"][0] = 0, 0   # tokens 0 .. 4 go by row 0
    leaves = {k: v.clone().requires_grad_() for k, v in dict(x=t["x"], y=t["y"], **{k: v for k, v in p.items() if v is not None}).items()}
    r, h = residual_norm(**leaves, post=post, pre="layer", tokens_per_row=5, eps=0.0)
    assert (r[4] == 0).all() and h[4].isnan().all()
    grads = dict(zip(leaves, torch.autograd.grad(r, list(leaves.values()), t["d_r"])))
    how = dict(y=t["y"], gate=p["gate"], post_weight=p["post_weight"], post=post, pre="none", tokens_per_row=5, eps=0.0)
    _, _, stats = mg.moga_residual_norm_fwd(t["x"], **how)
    want = mg.moga_residual_norm_bwd(t["d_r"], None, t["x"], stats, **how)
    for k, g in grads.items():
        assert torch.equal(g, torch.zeros_like(leaves[k]) if k in ("weight", "bias", "scale", "shift") else getattr(want, "d_" + k)), k


def test_outputs_that_nothing_comes_of():
    class Stop(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            return t.clone()

        @staticmethod
        def backward(ctx, g):
            return None

    x = torch.zeros((3, 72), device="cuda", requires_grad=True)
    w = torch.ones(72, device="cuda", requires_grad=True)
    r, h = residual_norm(x, x * 0, weight=w, pre="rms", eps=0.0)
    (x.sum() + Stop.apply(r).sum() + Stop.apply(h).sum()).backward()
    assert (x.grad == 1).all() and w.grad is None


def test_refuses():
    t, p = _inputs(8, 64, F32, BF, 1, each=4)
    how = dict(y=t["y"], **p, post="rms", pre="layer", tokens_per_row=4)
    call = lambda x=t["x"], **kw: mg.moga_residual_norm_fwd(x, **{**how, **kw})
    call()
    with pytest.raises(ValueError):
        call(gate=p["gate"][:1])
    with pytest.raises(ValueError):
        call(tokens_per_row=0)
    with pytest.raises(ValueError):
        call(weight=p["weight"][:32].contiguous())
    with pytest.raises(TypeError):
        call(shift=p["shift"].bfloat16())
    with pytest.raises(ValueError):
        call(post="other")
    with pytest.raises(ValueError):
        call(y=t["y"][:4].contiguous())
    with pytest.raises(AssertionError):
        call(x=t["x"].t())
    with pytest.raises(AssertionError):
        call(weight=p["weight"].cpu())
    with pytest.raises(mg.MogaError):
        call(x=t["x"].bfloat16(), y=t["y"].float())
    with pytest.raises(TypeError):
        call(x=t["x"].half())
    with pytest.raises(mg.MogaError):
        call(eps=float("nan"))
    with pytest.raises(mg.MogaError):
        call(post="none")   # with a weight of it
    with pytest.raises(mg.MogaError):
        mg.moga_residual_norm_fwd(t["x"], pre="none")
    _, _, stats = call()
    with pytest.raises(mg.MogaError):
        mg.moga_residual_norm_bwd(t["d_r"], None, t["x"], stats, **how)
    with pytest.raises(ValueError):
        mg.moga_residual_norm_bwd(t["d_r"], t["d_h"], t["x"], stats[:2].contiguous(), **how)
    with pytest.raises(TypeError):
        mg.moga_residual_norm_bwd(t["d_r"].bfloat16(), t["d_h"], t["x"], stats, **how)
