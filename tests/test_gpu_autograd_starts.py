"""autograd's rotary and moga_diff_attention on tensors that begin at any element, as pieces of longer ones do, and rotary of queries or keys alone."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import moga_diff_attention, rotary

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def _rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _later(t, by=3):
    """The same values, `by` elements behind the start of an allocation."""
    out = torch.cat([t.new_zeros(by), t.reshape(-1)])[by:].view(t.shape)
    assert out.is_contiguous() and out.data_ptr() % 16
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("maps", [1, 2])
def test_rotary(dtype, maps):
    N, D = 21, 64
    q, k, dq, dk = (_rnd(i, N, 2, D).to(dtype) for i in range(4))
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D // maps)
    a, b = _later(q).requires_grad_(), _later(k).requires_grad_()
    y = rotary(a, b, _later(pos), _later(freq, 1), maps=maps)
    assert all(torch.equal(s, t) for s, t in zip(y, mg.moga_rotary_fwd(q, k, pos, freq, maps=maps)))
    got = torch.autograd.grad(y, [a, b], [_later(dq), _later(dk)])
    assert all(torch.equal(s, t) for s, t in zip(got, mg.moga_rotary_bwd(dq, dk, pos, freq, maps=maps)))


def test_rotary_of_one_side():
    N, D = 33, 64
    x, d = _rnd(1, N, 3, D), _rnd(2, N, 3, D)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D)
    want, back = mg.moga_rotary_fwd(x, None, pos, freq)[0], mg.moga_rotary_bwd(d, None, pos, freq)[0]
    for side in range(2):
        a = x.clone().requires_grad_()
        y = rotary(*((a, None) if side == 0 else (None, a)), pos, freq)
        assert y[1 - side] is None and torch.equal(y[side], want)
        assert torch.equal(torch.autograd.grad(y[side], a, d)[0], back)
    with pytest.raises(ValueError):
        rotary(None, None, pos, freq)
    q, k = x.clone().requires_grad_(), d   # only one of two needs a gradient
    yq, yk = rotary(q, k, pos, freq)
    assert torch.equal(torch.autograd.grad(yq.sum() + yk.sum(), q)[0], mg.moga_rotary_bwd(torch.ones_like(x), None, pos, freq)[0])


@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)])
def test_differential_attention(dtype, D, positions):
    N, H, M = 150, 2, 3
    t = [_rnd(1, N, 64).to(dtype), _rnd(2, M, 64), *(_rnd(i, N, H, D).to(dtype) for i in (3, 4, 5)), _rnd(6, H)]
    d = _rnd(7, N, H, D).to(dtype)
    how = {}
    if positions:
        how = dict(positions=torch.arange(N, dtype=torch.int32, device="cuda"), inv_freq=mg.moga_rotary_freqs(D // 2)[0])

    def step(leaves):
        o, loss, group = moga_diff_attention(*leaves, 0.125, 0.1, True, **how)
        return [o, loss, group, *torch.autograd.grad([o, loss], leaves, [d, torch.ones_like(loss)])]

    want = step([a.clone().requires_grad_() for a in t])
    got = step([_later(a).requires_grad_() for a in t])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
