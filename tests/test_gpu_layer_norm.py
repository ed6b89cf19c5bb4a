"""Layer norm, forward and backward, against 64 bits.

Bounds (u = 2^-24): a mean is a sum of C values in pieces of at most 64 with 10 more steps, and so is the sum of squares: 80 u of the mean size of
what is summed; centring by it and the factor 1 / sqrt make that 160 u (|x - mu| + |mu| + max |x|) rstd for xh.  Sums over rows: pieces of at most
N rows, 80 more steps.  Then half a step of the output's type."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import layer_norm

from . import block_ref as ref

pytestmark = pytest.mark.gpu
U = ref.U
TYPES = [torch.bfloat16, torch.float32]


def _inputs(N, C, dtype, seed, affine=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, dy = (rnd(N, C) * 1.5 + 0.25).to(dtype), rnd(N, C).to(dtype)
    return x, dy, (rnd(C) + 1 if affine else None), (rnd(C) if affine else None)


def _check(x, dy, w, b, eps, y, mean, rstd, dx, dw, db):
    X, G = x.double(), dy.double()
    W = None if w is None else w.double()
    rows, C = X.shape
    half = ref.HALF_STEP[x.dtype]
    r_y, mu, r, xh = ref.norm_fwd(X, W, None if b is None else b.double(), eps)
    r_dx, r_dw, r_db = ref.norm_bwd(G, X, W, eps)
    size = X.abs().amax(1, keepdim=True)
    e_xh = 160 * U * r * size * (1 + r * size)
    aw = 1.0 if W is None else W.abs()
    ref.within(mean, mu[:, 0], 80 * U * size[:, 0], "mean")
    ref.within(rstd, r[:, 0], 160 * U * r[:, 0] * (1 + (r * size)[:, 0] ** 2), "rstd")
    ref.within(y, r_y, half * r_y.abs() + e_xh * aw + 4 * U * (xh.abs() * aw + (0 if b is None else b.double().abs())), "y")
    g = G.abs() * aw
    m0, m1 = g.mean(1, keepdim=True), (g * xh.abs()).mean(1, keepdim=True)
    e_dx = r * (e_xh * (m1 * 2 + (g * 1.0).mean(1, keepdim=True) * xh.abs()) + 160 * U * (g + m0 + xh.abs() * m1) * (1 + (r * size) ** 2))
    ref.within(dx, r_dx, half * r_dx.abs() + e_dx, "dx")
    if dw is not None:
        ref.within(dw, r_dw, (G.abs() * (e_xh + (rows + 80) * U * xh.abs())).sum(0) + U * r_dw.abs(), "dw")
        ref.within(db, r_db, (rows + 80) * U * G.abs().sum(0), "db")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,C", [(1, 1), (3, 2), (1, 5120), (5, 7), (17, 8), (33, 63), (64, 64), (9, 65), (1000, 128), (257, 129), (40, 255),
                                 (70, 512), (31, 1000), (19, 1535), (12, 1536), (65, 2047), (50, 2049), (7, 4097), (300, 5120), (6, 8191), (3, 8193),
                                 (4, 12289), (5, 16384)])
def test_forward_and_backward(N, C, dtype):
    x, dy, w, b = _inputs(N, C, dtype, 7 * N + C)
    eps = 1e-5
    y, mean, rstd = mg.moga_layer_norm_fwd(x, w, b, eps)
    dx, dw, db = mg.moga_layer_norm_bwd(dy, x, w, mean, rstd)
    if C == 1:   # a row of one value is its own mean
        assert torch.equal(y.float(), b.to(dtype).float().expand(N, 1)) and (dx == 0).all()
        return
    _check(x, dy, w, b, eps, y, mean, rstd, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,C", [(100, 128), (11, 1000), (77, 5120)])
def test_without_weights_and_without_statistics(N, C, dtype):
    x, dy, _, _ = _inputs(N, C, dtype, 11, affine=False)
    y, mean, rstd = mg.moga_layer_norm_fwd(x)
    dx, dw, db = mg.moga_layer_norm_bwd(dy, x, None, mean, rstd, want_dw=False)
    assert dw is None and db is None
    _check(x, dy, None, None, 1e-6, y, mean, rstd, dx, None, None)
    again, none, _ = mg.moga_layer_norm_fwd(x, want_stats=False)
    assert none is None and torch.equal(again, y)


@pytest.mark.parametrize("C", [96, 1536, 5000])
def test_weight_alone_and_bias_alone(C):
    x, dy, w, b = _inputs(20, C, torch.float32, 5)
    ones, zeros = torch.ones_like(w), torch.zeros_like(b)
    assert torch.equal(mg.moga_layer_norm_fwd(x, w, None)[0], mg.moga_layer_norm_fwd(x, w, zeros)[0])
    assert torch.equal(mg.moga_layer_norm_fwd(x, None, b)[0], mg.moga_layer_norm_fwd(x, ones, b)[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_of_heads_and_repeated_bits(dtype):
    x, dy, w, b = _inputs(70001, 128, dtype, 3)
    y, mean, rstd = mg.moga_layer_norm_fwd(x, w, b, 1e-6)
    dx, dw, db = mg.moga_layer_norm_bwd(dy, x, w, mean, rstd)
    _check(x, dy, w, b, 1e-6, y, mean, rstd, dx, dw, db)
    for _ in range(3):
        again = mg.moga_layer_norm_bwd(dy, x, w, mean, rstd)
        assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


def test_no_rows_and_constant_rows():
    x = torch.empty((0, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    y, mean, rstd = mg.moga_layer_norm_fwd(x, w, w)
    dx, dw, db = mg.moga_layer_norm_bwd(x, x, w, mean, rstd)
    assert y.shape == dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()
    x = torch.full((5, 1000), 3.0, device="cuda")
    y, mean, rstd = mg.moga_layer_norm_fwd(x, None, None, 1e-4)
    assert (y == 0).all() and (mean == 3).all() and torch.allclose(rstd, torch.full_like(rstd, 100.0))


@pytest.mark.parametrize("C", [128, 1536, 5120])
def test_large_offset(C):
    """The centred squares are summed, not squares less a square: a mean of 1,000 deviations costs bits of x, not of the variance."""
    x = torch.randn((30, C), device="cuda") + 1000.0
    y, mean, rstd = mg.moga_layer_norm_fwd(x)
    r, mu, rs, _ = ref.norm_fwd(x.double(), None, None, 1e-6)
    # the mean is off by at most 80 u 1,005, the centred value by that and half a step of itself
    ref.within(y, r, 200 * U * 1005 * rs * (1 + r.abs()), "y")


def test_a_row_with_infinities_does_not_touch_the_others():
    x, dy, w, b = _inputs(40, 200, torch.float32, 9)
    y0, m0, r0 = mg.moga_layer_norm_fwd(x, w, b)
    dx0, _, _ = mg.moga_layer_norm_bwd(dy, x, w, m0, r0)
    x[7, 3], x[20, 0] = float("inf"), float("nan")
    y, m, r = mg.moga_layer_norm_fwd(x, w, b)
    dx, _, _ = mg.moga_layer_norm_bwd(dy, x, w, m, r)
    keep = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(dx[keep], dx0[keep])
    assert y[20].isnan().all() and y[7].isnan().any()


def test_autograd():
    x, dy, w, b = _inputs(6 * 5, 96, torch.float32, 13)
    for wants in ((True, True, True), (True, False, False), (True, True, False), (True, False, True), (False, True, True)):
        xs, ws, bs = x.view(6, 5, 96).clone().requires_grad_(wants[0]), w.clone().requires_grad_(wants[1]), b.clone().requires_grad_(wants[2])
        y = layer_norm(xs, ws, bs, 1e-5)
        y.backward(dy.view(6, 5, 96))
        y2, mean, rstd = mg.moga_layer_norm_fwd(x, w, b, 1e-5)
        dx, dw, db = mg.moga_layer_norm_bwd(dy, x, w, mean, rstd)
        assert torch.equal(y.view(30, 96), y2)
        for t, want, r in ((xs, wants[0], dx.view(6, 5, 96)), (ws, wants[1], dw), (bs, wants[2], db)):
            assert torch.equal(t.grad, r) if want else t.grad is None
    # without weights; a gradient that is not contiguous
    xs = x.clone().requires_grad_(True)
    layer_norm(xs).backward(dy.t().contiguous().t())
    _, mean, rstd = mg.moga_layer_norm_fwd(x)
    assert torch.equal(xs.grad, mg.moga_layer_norm_bwd(dy, x, None, mean, rstd, want_dw=False)[0])
    # bias alone
    bs = b.clone().requires_grad_(True)
    layer_norm(x, None, bs).backward(dy)
    assert torch.equal(bs.grad, db)


def test_autograd_of_parts_of_longer_tensors():
    """Rows, weights and gradients that begin at an odd element."""
    C, n = 35, 9
    x, dy, w, b = _inputs(2 * n, C, torch.float32, 21)
    both = torch.cat([w, b]).requires_grad_(True)   # b begins at element 35
    xs = x.clone().requires_grad_(True)
    y = torch.cat([layer_norm(xs[:n], both[:C], both[C:], 1e-5), layer_norm(xs[n:], both[C:], both[:C], 1e-5)])
    y.backward(dy)
    parts = []
    for r, ww, bb in ((slice(0, n), w, b), (slice(n, 2 * n), b, w)):
        xr = x[r].clone()
        yr, mean, rstd = mg.moga_layer_norm_fwd(xr, ww, bb, 1e-5)
        assert torch.equal(y[r], yr)
        parts.append(mg.moga_layer_norm_bwd(dy[r].clone(), xr, ww, mean, rstd))
    assert torch.equal(xs.grad, torch.cat([p[0] for p in parts]))
    assert torch.equal(both.grad, torch.cat([parts[0][1] + parts[1][2], parts[0][2] + parts[1][1]]))


def test_refuses_tensors_that_do_not_fit():
    x, dy, w, b = _inputs(8, 64, torch.bfloat16, 1)
    with pytest.raises(ValueError):
        mg.moga_layer_norm_fwd(x, w[:32].contiguous(), b)
    with pytest.raises(TypeError):
        mg.moga_layer_norm_fwd(x, w.bfloat16(), b)
    with pytest.raises(AssertionError):
        mg.moga_layer_norm_fwd(x.t(), w, b)
    with pytest.raises(TypeError):
        mg.moga_layer_norm_fwd(x.half(), w, b)
    with pytest.raises(ValueError):
        mg.moga_layer_norm_fwd(x.view(-1), w, b)
    with pytest.raises(mg.MogaError):
        mg.moga_layer_norm_fwd(x, w, b, eps=-1.0)
    y, mean, rstd = mg.moga_layer_norm_fwd(x, w, b)
    with pytest.raises(TypeError):
        mg.moga_layer_norm_bwd(dy.float(), x, w, mean, rstd)
    with pytest.raises(ValueError):
        mg.moga_layer_norm_bwd(dy, x, w, mean[:4].contiguous(), rstd)
