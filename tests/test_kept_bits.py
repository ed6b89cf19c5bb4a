"""The a and u that the bf16 feed-forward keeps for its backward (bf16 and two more bits each), taken apart on the host; no GPU."""
import pytest
import torch

from . import block_parts_ref as ref
from .block_ref import U

BF = torch.bfloat16


def step(v):
    """Of bf16, at v."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -100))) - 7)


def value(rounded, bits):
    """bits - 1 quarters of a step on from the rounded value (below a power of two the steps are half as long), in fp32's bits."""
    return (rounded.float().view(torch.int32) + (bits.int() - 1) * 0x4000).view(torch.float32).double()


def parts(au, N, F):
    """What the forward kept -> rounded a and u, their bits: each [N, F] in 64 bits."""
    r = au[:2 * N * F].view(N, 2, F).double()
    b = au[2 * N * F:].view(torch.uint8).view(N, F // 2)
    pairs = torch.stack([b & 15, b >> 4], -1).view(N, F)
    return r[:, 0], r[:, 1], (pairs & 3).double(), (pairs >> 2).double()


def off(got, a, u, bits_a, bits_u, act):
    """How far [da, du] of dh = 1 are off, the worst as a part of what they may be: half a step of their own, and what the activation's fp32 is off by
    (its bounds in ref.gated_ffn; 2^-23 more for the products).  Both values' steps are asked: one may lie across a power of two."""
    a, u = value(a, bits_a), value(u, bits_u)
    f, slope = ref.activation(a, act)
    cube = 64 * U * (1 + a.abs()) ** 3
    e_f = 8 * U * (2 + a.abs()) * a.abs() + cube * (act == "gelu_tanh")
    want = torch.cat([u * slope, f], 1)
    e = torch.cat([u.abs() * cube, e_f], 1) + 2 * U * want.abs()
    got = got.double()
    return float(((got - want).abs() / (torch.maximum(step(got), step(want)) / 2 + e)).max())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("N,F", [(5, 264), (300, 264)])
def test_off_tells_wrong_bits(N, F, act):
    """A backward that makes anything else of the bits is off by more than its rounding."""
    g = torch.Generator().manual_seed(N)
    a, u = (torch.randn((N, F), generator=g, dtype=torch.float64) * 1.5 for _ in range(2))
    ra, ru = a.to(BF).double(), u.to(BF).double()
    bits = lambda v, r: ((v.float().view(torch.int32) - r.float().view(torch.int32) + 0x6000) >> 14).clamp(0, 3).double()
    ba, bu = bits(a, ra), bits(u, ru)
    assert ((value(ra, ba) - a).abs() <= step(ra) / 4 * 1.001).all()

    def made(bits_a, bits_u):
        x, y = value(ra, bits_a), value(ru, bits_u)
        f, slope = ref.activation(x, act)
        return torch.cat([y * slope, f], 1).to(BF)
    right = made(ba, bu)
    assert off(right, ra, ru, ba, bu, act) <= 1
    beside = lambda b: b.view(N, F // 2, 2).flip(-1).reshape(N, F)
    one = torch.ones_like(ba)
    for wrong in ((one, one), (bu, ba), (beside(ba), beside(bu)), (0 * one, 0 * one), (3 * one, 3 * one), (ba, one), (one, bu), (ba.roll(1, 0), bu.roll(1, 0)), (ba.roll(8, 1), bu.roll(8, 1)),
                  (3 - ba, 3 - bu)):
        assert off(made(*wrong), ra, ru, ba, bu, act) > 1.1
