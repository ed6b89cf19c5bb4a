"""moga_diff_attention without a gradient keeps nothing for one: the two maps' sums of V are written only where a backward will read them."""
import pytest
import torch

from paper_2510_18692_amd.autograd import moga_diff_attention

pytestmark = pytest.mark.gpu


def _inputs(N, H, D=128):
    g = torch.Generator(device="cuda").manual_seed(N)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, v = (rnd(N, H, D).bfloat16() for _ in range(3))
    return rnd(N, 32).bfloat16(), rnd(8, 32), q, k, v, torch.full((H,), 0.4, device="cuda")


def _peak(run):
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = run()
    torch.cuda.synchronize()
    return out, torch.cuda.max_memory_allocated() - before


@pytest.mark.parametrize("how", ["no_grad", "inference_mode", "no leaf"])
def test_no_gradient_no_maps(how):
    N, H = 20000, 12
    t = _inputs(N, H)
    rows = t[2].nbytes                      # q, k and v in sorted order, the output in both orders: 5 of them; the maps' sums in fp32 are 4
    guard = {"no_grad": torch.no_grad(), "inference_mode": torch.inference_mode(), "no leaf": torch.enable_grad()}[how]
    if how != "no leaf":
        t[5].requires_grad_()
    with guard:
        (o, _, _), peak = _peak(lambda: moga_diff_attention(*t, 0.125))
    assert 5 * rows <= peak < 7 * rows, (peak / rows)
    assert not o.requires_grad
    t[5].requires_grad_()
    (want, _, _), peak = _peak(lambda: moga_diff_attention(*t, 0.125))
    assert peak >= 9 * rows and torch.equal(o, want.detach())


@pytest.mark.parametrize("leaf", range(1, 6))
def test_one_leaf_is_enough_for_a_backward(leaf):
    N, H = 300, 2
    t = list(_inputs(N, H))
    all_of_them = [a.clone().requires_grad_(i > 0) for i, a in enumerate(t)]
    o, _, _ = moga_diff_attention(*all_of_them, 0.125)
    o.float().square().sum().backward()
    t[leaf].requires_grad_()
    o, _, _ = moga_diff_attention(*t, 0.125)
    o.float().square().sum().backward()
    assert torch.equal(t[leaf].grad, all_of_them[leaf].grad)


def test_frequencies_that_ask_for_a_gradient():
    """They get none, but autograd runs the backward for them."""
    from paper_2510_18692_amd import binding as mg
    N, H = 200, 2
    t = _inputs(N, H)
    freq = mg.moga_rotary_freqs(64)[0].requires_grad_()
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    o, _, _ = moga_diff_attention(*t, 0.125, positions=pos, inv_freq=freq)
    o.float().sum().backward()
    assert freq.grad is None
