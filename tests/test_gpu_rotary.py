"""Rotary positions against 64 bits.

Bound (u = 2^-24): the part of a turn is rounded to fp32 (at most 2^-25 of a turn, 3.2 u radians), sine and cosine are within 2 u of it, and two
products, a sum and the factor add 4 u: 10 u factor (|x1| + |x2|) for a result; then half a step of its type."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import rotary

from . import block_ref as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def _rnd(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _close(got, x, pos, freq, pairs, inter, factor, sign, what):
    r = ref.rotate(x.double(), pos, freq, pairs, inter, factor, sign)
    turned = torch.zeros_like(r)
    turned[..., :2 * freq.numel()] = 1
    bound = turned * 10 * ref.U * abs(factor) * ref.pair_sizes(x.double(), 2 * freq.numel(), inter) + turned * ref.HALF_STEP[x.dtype] * r.abs()
    ref.within(got, r, bound, what)


CASES = [   # N, Hq, Hk, D, R
    (1, 1, 1, 128, 128), (1, 40, 40, 128, 128), (3, 12, 4, 128, 96), (50, 3, 3, 128, 124), (17, 2, 1, 64, 62), (129, 5, 2, 64, 64), (33, 4, 4, 64, 2),
    (40, 2, 2, 8, 6), (23, 1, 3, 24, 10), (20, 2, 2, 256, 256), (1001, 12, 12, 128, 128), (700, 3, 1, 40, 36)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,D,R", CASES)
def test_token_order(N, Hq, Hk, D, R, inter, dtype):
    q, k = _rnd(1, N, Hq, D, dtype=dtype), _rnd(2, N, Hk, D, dtype=dtype)
    freq, factor = mg.moga_rotary_freqs(R, scaling="parts", scale_factor=8.0, original_len=2048)
    pos = torch.randint(-5000, 600000, (N,), generator=torch.Generator().manual_seed(N), dtype=torch.int32).cuda()
    for f, sign in ((mg.moga_rotary_fwd, 1), (mg.moga_rotary_bwd, -1)):
        yq, yk = f(q, k, pos, freq, interleaved=inter, factor=factor)
        _close(yq, q, pos[None], freq, [R // 2], inter, factor, sign, "q")
        _close(yk, k, pos[None], freq, [R // 2], inter, factor, sign, "k")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dims", [(44, 42, 42), (128, 0), (0, 64), (16, 16, 16, 16), (2, 4, 6)])
def test_axes_and_sorted_order(dims, inter, dtype):
    N, H, D = 517, 3, 128
    q, k, v = (_rnd(i, N, H, D, dtype=dtype) for i in (3, 4, 5))
    freq, _ = mg.moga_rotary_freqs(list(dims))
    pairs = [d // 2 for d in dims]
    pos = torch.randint(0, 3000, (len(dims), N), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    how = dict(axis_pairs=pairs, interleaved=inter, factor=1.0)
    yq, yk = mg.moga_rotary_fwd(q, k, pos, freq, **how)
    _close(yq, q, pos, freq, pairs, inter, 1.0, 1, "q")
    group = torch.randint(0, 7, (N,), generator=torch.Generator().manual_seed(8), dtype=torch.int32).cuda()
    plain = mg.moga_permute(group, 7, yq, yk, v)
    sorted_ = mg.moga_rotary_permute_fwd(q, k, v, plain["perm"], pos, freq, **how)
    for got, name in zip(sorted_, ("qh", "kh", "vh")):
        assert torch.equal(got, plain[name]), name   # the bits of the two calls
    back = mg.moga_rotary_permute_bwd(*sorted_, plain["perm"], pos, freq, **how)
    two = mg.moga_permute_bwd(*sorted_, plain["perm"])
    dq, dk = mg.moga_rotary_bwd(two[0], two[1], pos, freq, **how)
    assert torch.equal(back[0], dq) and torch.equal(back[1], dk) and torch.equal(back[2], v)


@pytest.mark.parametrize("N,H,D,R", [(1, 1, 128, 128), (2, 40, 128, 128), (5, 3, 128, 92), (4099, 12, 128, 64), (63, 2, 64, 60)])
def test_sorted_order_at_odd_sizes(N, H, D, R):
    dtype = torch.bfloat16
    q, k, v = (_rnd(i, N, H, D, dtype=dtype) for i in (3, 4, 5))
    freq, _ = mg.moga_rotary_freqs(R)
    pos = torch.arange(N, dtype=torch.int32).cuda()
    perm = torch.randperm(N, generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    qh, kh, vh = mg.moga_rotary_permute_fwd(q, k, v, perm, pos, freq)
    yq, yk = mg.moga_rotary_fwd(q, k, pos, freq)
    for got, y in ((qh, yq), (kh, yk), (vh, v)):
        assert torch.equal(got, y[perm.long()].transpose(0, 1))


def test_far_positions_and_the_ends_of_the_range():
    N, R = 64, 128
    q = _rnd(1, N, 2, 128)
    freq, _ = mg.moga_rotary_freqs(R)
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 16777217, 580319, 0, 1, -1] * 8, dtype=torch.int32).cuda()
    y, _ = mg.moga_rotary_fwd(q, None, pos, freq)
    # at 2^31 the product in 64 bits is off by some 2^-22 radians in the reference and the kernel alike: 8 u more
    r = ref.rotate(q.double(), pos[None], freq, [64], False, 1.0)
    ref.within(y, r, 18 * ref.U * ref.pair_sizes(q.double(), R, False), "y")
    turned = mg.moga_rotary_fwd(q, None, torch.zeros_like(pos), freq)[0]
    assert torch.equal(turned, q)   # position 0


def test_backward_is_the_transpose_and_norms_stay():
    N, D = 300, 64
    q, d = _rnd(1, N, 4, D), _rnd(2, N, 4, D)
    pos = torch.arange(N, dtype=torch.int32).cuda() * 97
    freq, _ = mg.moga_rotary_freqs(48)
    y, _ = mg.moga_rotary_fwd(q, None, pos, freq, factor=1.5)
    b, _ = mg.moga_rotary_bwd(d, None, pos, freq, factor=1.5)
    lhs, rhs = (y.double() * d.double()).sum(), (q.double() * b.double()).sum()
    assert abs(lhs - rhs) <= 40 * ref.U * (q.double().abs() * d.double().abs()).sum() * 3
    y, _ = mg.moga_rotary_fwd(q, None, pos, freq)
    assert torch.allclose(y.norm(dim=2), q.norm(dim=2), rtol=1e-6)


def test_infinities_stay_in_their_pair():
    q = _rnd(1, 10, 2, 128)
    q[3, 1, 127], q[4, 0, 100] = float("inf"), float("nan")   # behind the rotated part: copied
    pos = torch.arange(10, dtype=torch.int32).cuda()
    for R, inter in ((96, False), (92, False), (96, True), (90, True)):
        freq, _ = mg.moga_rotary_freqs(R)
        y, _ = mg.moga_rotary_fwd(q, None, pos, freq, interleaved=inter)
        assert torch.equal(y[..., R:].nan_to_num(7.0, 8.0), q[..., R:].nan_to_num(7.0, 8.0)) and y[..., :R].isfinite().all()


def test_autograd():
    N = 70
    q, k, dq, dk = _rnd(1, N, 4, 64), _rnd(2, N, 2, 64), _rnd(3, N, 4, 64), _rnd(4, N, 2, 64)
    pos = torch.arange(N, dtype=torch.int32).cuda()
    freq, _ = mg.moga_rotary_freqs(64)
    a, b = q.clone().requires_grad_(True), k.clone().requires_grad_(True)
    yq, yk = rotary(a, b, pos, freq, interleaved=True)
    gq, gk = torch.autograd.grad([yq, yk], [a, b], [dq, dk])
    eq, ek = mg.moga_rotary_bwd(dq, dk, pos, freq, interleaved=True)
    assert torch.equal(gq, eq) and torch.equal(gk, ek)
    yq, yk = rotary(a, b, pos, freq, interleaved=True)   # one of the two alone
    assert torch.equal(torch.autograd.grad(yk, b, dk)[0], ek)


def test_autograd_at_positions_of_a_piece():
    """Positions that are a slice of a longer list begin at any element."""
    q, k, d = _rnd(1, 21, 2, 64), _rnd(2, 21, 1, 64), _rnd(3, 21, 2, 64)
    pos = torch.arange(100, dtype=torch.int32).cuda()
    freq, _ = mg.moga_rotary_freqs(64)
    a = q.clone().requires_grad_(True)
    yq, yk = rotary(a, k, pos[37:58], freq)
    eq, ek = mg.moga_rotary_fwd(q, k, pos[37:58].clone(), freq)
    assert torch.equal(yq, eq) and torch.equal(yk, ek)
    assert torch.equal(torch.autograd.grad(yq, a, d)[0], mg.moga_rotary_bwd(d, None, pos[37:58].clone(), freq)[0])


def test_nothing_to_do_and_refusals():
    freq, _ = mg.moga_rotary_freqs(128)
    e = torch.empty((0, 3, 128), device="cuda")
    y, _ = mg.moga_rotary_fwd(e, None, torch.empty(0, dtype=torch.int32, device="cuda"), freq)
    assert y.shape == e.shape
    q, pos = _rnd(1, 6, 2, 128), torch.arange(6, dtype=torch.int32).cuda()
    with pytest.raises(ValueError):
        mg.moga_rotary_fwd(None, None, pos, freq)
    with pytest.raises(ValueError):
        mg.moga_rotary_fwd(q, None, pos[:5].contiguous(), freq)
    with pytest.raises(TypeError):
        mg.moga_rotary_fwd(q, None, pos.long(), freq)
    with pytest.raises(TypeError):
        mg.moga_rotary_fwd(q, None, pos, freq.float())
    with pytest.raises(ValueError):
        mg.moga_rotary_fwd(q, None, pos[None].repeat(3, 1), freq)          # three axes, no axis_pairs
    with pytest.raises(mg.MogaError):
        mg.moga_rotary_fwd(q, None, pos[None].repeat(2, 1), freq, axis_pairs=[32, 31])
    with pytest.raises(mg.MogaError):
        mg.moga_rotary_fwd(q[..., :64].contiguous(), None, pos, freq)      # more pairs than the head has
    with pytest.raises(TypeError):
        mg.moga_rotary_fwd(q, q.bfloat16(), pos, freq)
