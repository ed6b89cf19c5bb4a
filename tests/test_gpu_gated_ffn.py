"""The gated feed-forward, forward and backward, against 64 bits; bounds in block_parts_ref."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import gated_ffn

from . import block_parts_ref as ref
from .block_ref import within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _inputs(N, C, F, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda s, *n: (torch.randn(n, generator=g, device="cuda") * s).to(dtype)
    return rnd(1.0, N, C), rnd(1.5 * C ** -0.5, 2 * F, C), rnd(F ** -0.5, C, F), rnd(1.0, N, C)


def _check(N, C, F, dtype, act, seed=0):
    x, wi, wo, dy = _inputs(N, C, F, dtype, 7 * N + C + F + seed)
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, act)
    d_x, d_wi, d_wo = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, act)
    want = ref.gated_ffn(x, wi, wo, act, dy)
    got = dict(y=y, au=au[:2 * N * F].view(N, 2 * F), h=h, d_x=d_x, d_w_in=d_wi, d_w_out=d_wo)
    for k, v in got.items():
        within(v, *want[k], k)
    alone, none, _ = mg.moga_gated_ffn_fwd(x, wi, wo, act, want_saved=False)
    assert none is None and torch.equal(alone, y)
    return (x, wi, wo, dy), got


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("N,C,F", [(1, 8, 8), (2, 1536, 264), (3, 16, 24), (16, 72, 128), (17, 136, 40), (33, 264, 1032), (64, 512, 1368), (65, 264, 520),
                                   (100, 1536, 512), (129, 128, 4104), (300, 264, 200), (1563, 136, 264), (1030, 520, 264), (4099, 64, 136)])
def test_bf16(N, C, F, act):
    _check(N, C, F, BF, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("N,C,F", [(1, 4, 4), (1, 512, 1368), (5, 12, 20), (31, 100, 36), (70, 100, 36), (257, 132, 260), (1000, 64, 300), (5003, 36, 64)])
def test_f32(N, C, F, act):
    _check(N, C, F, F32, act)


@pytest.mark.parametrize("dtype,N,C,F", [(BF, 20000, 128, 264), (BF, 9001, 520, 136), (BF, 300, 264, 16392), (F32, 9001, 132, 68), (BF, 2600, 1032, 1544), (BF, 2126, 1296, 1936),
                                         (BF, 4601, 1544, 3104), (F32, 541, 792, 3128)])
def test_long_sums_and_repeated_bits(dtype, N, C, F):
    (x, wi, wo, dy), got = _check(N, C, F, dtype, "silu")
    for _ in range(3):
        y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo)
        d = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h)
        assert all(torch.equal(a, b) for a, b in zip((y, au[:2 * N * F].view(N, 2 * F), h, *d), got.values()))


@pytest.mark.parametrize("N", [1, 30, 130, 500, 3000])
def test_two_more_bits_of_a_and_u(N):
    """Behind the rounded a and u: their distance from the values in quarters of a step of bf16 (2^-7 of the power of two below), from -1/4 to 1/2.  What is
    put together is off by at most a quarter of a step, and by an eighth where the rounding went down by no more than three eighths."""
    C, F = 72, 136
    x, wi, wo, _ = _inputs(N, C, F, BF, 4)
    x[N // 2] = 0
    _, au, _ = mg.moga_gated_ffn_fwd(x, wi, wo)
    want, e = ref.gated_ffn(x, wi, wo, "silu")["au"]
    e = e - ref.HALF_STEP[BF] * want.abs()   # of the fp32 sums alone
    rounded = au[:2 * N * F].view(N, 2, F)
    b = au[2 * N * F:].view(torch.uint8).view(N, F // 2)
    pairs = torch.stack([b & 15, b >> 4], -1).view(N, F)
    bits = torch.stack([pairs & 3, pairs >> 2], 1).double()
    step = torch.exp2(torch.floor(torch.log2(rounded.double().abs().clamp(min=1e-30))) - 7)
    got = rounded.double() + torch.sign(rounded.double()) * step * (bits - 1) / 4
    off = (got - want.view(N, 2, F)).abs()
    assert (off <= step / 4 * 1.0001 + e.view(N, 2, F)).all()
    # uniform in [-1/2, 1/2] of a step: an eighth of them lie below -3/8, and are off by an eighth to a quarter
    assert (off <= step / 8 * 1.0001 + e.view(N, 2, F)).double().mean() > 0.8
    assert (rounded[N // 2] == 0).all() and (bits[N // 2] == 1).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N", [5, 40, 200, 700])
def test_bad_tokens_do_not_touch_the_others(dtype, N):
    C, F = 136, 264
    x, wi, wo, dy = _inputs(N, C, F, dtype, 3)
    y0, au0, h0 = mg.moga_gated_ffn_fwd(x, wi, wo)
    d0 = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au0, h0, want_dw_in=False, want_dw_out=False)[0]
    bad = [0, N // 2, N - 1]
    x[bad[0], C - 1], x[bad[1], 0], x[bad[2], 5] = float("nan"), float("inf"), -float("inf")
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo)
    d = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, want_dw_in=False, want_dw_out=False)[0]
    keep = [i for i in range(N) if i not in bad]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(d[keep], d0[keep]) and y[bad[0]].isnan().all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_arguments(act, dtype):
    """Arguments whose exponential overflows: act is a or 0, its derivative 1 or 0, nothing is NaN."""
    x = torch.zeros((6, 8), device="cuda", dtype=dtype)
    x[:, 0] = torch.tensor([1e4, -1e4, 3e18, -3e18, 1e2, -1e2], device="cuda")
    wi, wo = (torch.zeros(s, device="cuda", dtype=dtype) for s in ((16, 8), (8, 8)))
    wi[0, 0], wi[8, 0], wo[0, 0] = 1.0, 1.0, 1.0
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, act)
    a = x[:, 0].double()
    want = torch.where(a > 0, a, 0) * a
    within(h[:, 0], want, 4 * ref.HALF_STEP[dtype] * want, "h")
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    d_x, d_wi, d_wo = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, act)
    assert d_x.isfinite().all()
    within(d_x[:, 0], torch.where(a > 0, 2 * a, 0), 8 * ref.HALF_STEP[dtype] * a.abs(), "d_x")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_arguments_whose_square_overflows(act, dtype):
    """a = +-1e30 beside u = 1e-30: h is 1 or 0, and so are the derivatives by either, times the other."""
    x = torch.zeros((2, 8), device="cuda", dtype=dtype)
    x[:, 0], x[:, 1] = torch.tensor([1e15, -1e15], device="cuda"), 1e-15
    wi, wo = (torch.zeros(s, device="cuda", dtype=dtype) for s in ((16, 8), (8, 8)))
    wi[0, 0], wi[8, 1], wo[0, 0] = 1e15, 1e-15, 1.0
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, act)
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    d_x, d_wi, d_wo = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, act)
    e = 16 * ref.HALF_STEP[dtype]   # roundings of x, w, a, u, h and of the results
    on = torch.tensor([1.0, 0.0], device="cuda", dtype=torch.float64)
    within(h[:, 0], on, e * on, "h")
    within(d_x[:, 0], on * 1e-15, e * 1e-15 * on, "d_x by a")      # u act'(a) w
    within(d_x[:, 1], on * 1e15, e * 1e15 * on, "d_x by u")        # act(a) w
    assert y.isfinite().all() and d_x.isfinite().all() and d_wo.isfinite().all()
    assert not d_wi.isnan().any() and d_wi[8, 0].isinf()   # act(a) x is 1e30 * 1e15, past fp32's range


def test_lower_tail_of_gelu():
    """fp32, a = -2 .. -12 exactly: h and the gradients by a and by u, relative to themselves.  Phi(a) = erfc(z) / 2 with z = -a / sqrt 2 off by 2 u (the constant
    and the product), where d ln erfc / dz is below 2 z + 2 / z in size: 2 u (2 z^2 + 2) = (2 a^2 + 4) u, and 32 u (16 ulp) for erfc itself.  The density: its
    argument a^2 / 2 twice rounded, a^2 u, 4 u (2 ulp) for exp and 4 u for its products.  Products of the results and the derivative's sum: 8 u."""
    n = 41
    a = -2 - torch.arange(n, device="cuda", dtype=torch.float64) / 4
    x, wi, wo = (torch.zeros(s, device="cuda") for s in ((n, 4), (8, 4), (4, 4)))
    x[:, 0], x[:, 1] = a.float(), 1
    wi[0, 0], wi[4, 1], wo[0, 0] = 1, 1, 1
    _, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, "gelu")
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    d_x, _, _ = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, "gelu")
    u, phi, density = ref.U, torch.erfc(-a * 0.5 ** 0.5) / 2, torch.exp(-a * a / 2) * (2 * torch.pi) ** -0.5
    e_phi, e_density = (2 * a * a + 36) * u * phi, (a * a + 8) * u * density
    e_act = a.abs() * (e_phi + 8 * u * phi)
    within(h[:, 0], a * phi, e_act, "h")
    within(d_x[:, 1], a * phi, e_act, "by u")
    within(d_x[:, 0], phi + a * density, e_phi + 8 * u * phi + a.abs() * (e_density + 8 * u * density), "by a")


def test_parts_of_the_backward():
    x, wi, wo, dy = _inputs(300, 136, 264, BF, 1)
    _, au, h = mg.moga_gated_ffn_fwd(x, wi, wo)
    full = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h)
    for i, k in enumerate(("want_dx", "want_dw_in", "want_dw_out")):
        only = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, **{n: n == k for n in ("want_dx", "want_dw_in", "want_dw_out")})
        assert torch.equal(only[i], full[i]) and [v is None for v in only].count(True) == 2
    assert mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, want_dx=False, want_dw_in=False, want_dw_out=False) == (None, None, None)


def test_half_a_billion_tokens():
    """537,001,792 tokens, millions of blocks and tensors of more than 2^32 values.  The same rows over and over have the same results over and over (each sum
    is one step of k, whatever the tiles)."""
    n, times, C, F = 4099, 131008, 8, 8
    x, wi, wo, dy = _inputs(n, C, F, BF, 5)
    y0, au0, h0 = mg.moga_gated_ffn_fwd(x, wi, wo)
    d0 = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au0, h0, want_dw_in=False, want_dw_out=False)[0]
    many = lambda t: t.repeat(times, 1)
    big = many(x)
    y, au, h = mg.moga_gated_ffn_fwd(big, wi, wo)
    d = mg.moga_gated_ffn_bwd(many(dy), big, wi, wo, au, h, want_dw_in=False, want_dw_out=False)[0]
    for got, want in ((y, y0), (h, h0), (au[:2 * n * times * F].view(-1, 2 * F), au0[:2 * n * F].view(n, 2 * F)), (d, d0)):
        got, want = got.view(times, -1).view(torch.int64), want.reshape(-1).view(torch.int64)
        assert all((got[i:i + 4096] == want).all() for i in range(0, times, 4096))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_tokens(dtype):
    x, wi, wo, dy = _inputs(0, 16, 24, dtype, 1)
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo)
    d_x, d_wi, d_wo = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h)
    assert y.shape == d_x.shape == (0, 16) and d_wi.shape == wi.shape and d_wo.shape == wo.shape and (d_wi == 0).all() and (d_wo == 0).all()


def test_gradients_are_difference_quotients():
    """Along a random direction of each input (fp32: quotients to 2e-3 of the gradient's size)."""
    leaves = [t.requires_grad_() for t in _inputs(9, 20, 28, F32, 2)[:3]]
    dy = _inputs(9, 20, 28, F32, 2)[3]
    for act in ("silu", "gelu", "gelu_tanh"):
        f = lambda *v: (gated_ffn(*v, activation=act).double() * dy.double()).sum()
        for i, g in enumerate(torch.autograd.grad(f(*leaves), leaves)):
            v = [t.detach() for t in leaves]
            step = torch.randn_like(v[i])
            at = lambda e: float(f(*v[:i], v[i] + e * step, *v[i + 1:]))
            want = float((g.double() * step.double()).sum())
            assert abs((at(1e-2) - at(-1e-2)) / 2e-2 - want) <= 2e-3 * float(g.norm() * step.norm()), (act, i)


def test_autograd():
    x, wi, wo, dy = _inputs(60, 136, 72, BF, 6)
    xs, ws, os = (t.clone().requires_grad_() for t in (x, wi, wo))
    y = gated_ffn(xs.view(3, 20, 136), ws, os, "gelu")
    assert y.shape == (3, 20, 136)
    y.backward(dy.view(3, 20, 136))
    yr, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, "gelu")
    d = mg.moga_gated_ffn_bwd(dy, x, wi, wo, au, h, "gelu")
    assert torch.equal(y.view(60, 136), yr) and all(torch.equal(a.grad, b) for a, b in zip((xs, ws, os), d))
    # one leaf; tensors that begin anywhere; a gradient in another order; no graph
    flat = torch.cat([wi.view(-1)[:3], wi.view(-1)]).requires_grad_()
    gated_ffn(x, flat[3:].view(wi.shape), wo, "gelu").backward(dy.t().contiguous().t())
    assert torch.equal(flat.grad[3:].view(wi.shape), d[1])
    with torch.no_grad():
        again = gated_ffn(x, ws, wo, "gelu")
    assert torch.equal(again, yr) and not again.requires_grad
    with pytest.raises(RuntimeError, match="no second derivative"):
        g, = torch.autograd.grad(gated_ffn(xs, wi, wo).square().sum(), xs, create_graph=True)
        (g.square().sum() + xs.square().sum()).backward()


def test_refuses():
    x, wi, wo, dy = _inputs(8, 64, 32, BF, 1)
    y, au, h = mg.moga_gated_ffn_fwd(x, wi, wo)
    with pytest.raises(ValueError):
        mg.moga_gated_ffn_fwd(x, wi[:32].contiguous(), wo)
    with pytest.raises(ValueError):
        mg.moga_gated_ffn_fwd(x, wi, wo, "relu")
    with pytest.raises(TypeError):
        mg.moga_gated_ffn_fwd(x, wi.float(), wo)
    with pytest.raises(TypeError):
        mg.moga_gated_ffn_fwd(x.half(), wi.half(), wo.half())
    with pytest.raises(AssertionError):
        mg.moga_gated_ffn_fwd(x, wi, wo.t().contiguous().t())
    with pytest.raises(AssertionError):
        mg.moga_gated_ffn_fwd(x, wi, wo.cpu())
    with pytest.raises(mg.MogaError):
        mg.moga_gated_ffn_fwd(*_inputs(4, 12, 8, BF, 1)[:3])   # width no multiple of 8
    with pytest.raises(mg.MogaError):
        mg.moga_gated_ffn_fwd(*_inputs(4, 8, 12, BF, 1)[:3])
    with pytest.raises(ValueError):
        mg.moga_gated_ffn_bwd(dy, x, wi, wo, au[:-8].contiguous(), h)
    with pytest.raises(TypeError):
        mg.moga_gated_ffn_bwd(dy.float(), x, wi, wo, au, h)
