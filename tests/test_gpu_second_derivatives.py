"""Layer norm, rotary positions and differential attention have first derivatives.  A graph through their gradients refuses to be differentiated;
it does not leave their part out."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import layer_norm, moga_diff_attention, rotary

pytestmark = pytest.mark.gpu
N, H, D = 40, 2, 64


def _rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _norm():
    leaves = [_rnd(1, N, D).requires_grad_(), _rnd(2, D).requires_grad_(), _rnd(3, D).requires_grad_()]
    return leaves, lambda x, w, b: layer_norm(x, w, b)


def _norm_without_weights():
    return [_rnd(1, N, D).requires_grad_()], lambda x: layer_norm(x)


def _rotary():
    freq, _ = mg.moga_rotary_freqs(D)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    return [_rnd(1, N, H, D).requires_grad_(), _rnd(2, N, H, D).requires_grad_()], lambda q, k: sum(rotary(q, k, pos, freq))


def _diff():
    x = _rnd(5, N, 16)
    leaves = [_rnd(6, 3, 16), *(_rnd(i, N, H, D) for i in (1, 2, 3)), _rnd(4, H)]
    return [t.requires_grad_() for t in leaves], lambda w, q, k, v, lam: moga_diff_attention(x, w, q, k, v, lam, 0.125)[0]


@pytest.mark.parametrize("make", [_norm, _norm_without_weights, _rotary, _diff])
def test_refused(make):
    leaves, f = make()
    want = torch.autograd.grad(f(*leaves).square().sum(), leaves)
    got = torch.autograd.grad(f(*leaves).square().sum(), leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for t, g in zip(leaves, got):
        assert g.requires_grad
        with pytest.raises(RuntimeError, match="no second derivative"):
            # beside a part that has one: what silence would leave out
            torch.autograd.grad(g.square().sum() + t.square().sum(), t, retain_graph=True)


def test_gradients_alone_are_as_before():
    x = _rnd(1, N, D).requires_grad_()
    layer_norm(x).square().sum().backward()
    assert not x.grad.requires_grad


def test_rotation_is_linear():
    """Where nothing that the gradient depends on needs one, there is nothing to refuse."""
    freq, _ = mg.moga_rotary_freqs(D)
    pos, d = torch.arange(N, dtype=torch.int32, device="cuda"), _rnd(3, N, H, D)
    q, k = _rnd(1, N, H, D).requires_grad_(), _rnd(2, N, H, D)
    g, = torch.autograd.grad(rotary(q, k, pos, freq)[0], q, d, create_graph=True)
    assert not g.requires_grad and torch.equal(g, mg.moga_rotary_bwd(d, None, pos, freq)[0])
