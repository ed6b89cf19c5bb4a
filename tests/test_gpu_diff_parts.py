"""The output of differential attention does not depend on whether the two maps' sums are written beside it."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D,dtype", [(2, 64, torch.float32), (3, 128, torch.float32), (3, 128, torch.bfloat16)])
@pytest.mark.parametrize("sq,sk", [([64, 20, 40], None), ([500, 0, 700], None), ([2000, 1300, 2100], None), ([1, 1, 1], [5000, 300, 9000]), ([1, 40], [600, 900])])
def test_same_bits_with_and_without_parts(H, D, dtype, sq, sk):
    g = torch.Generator(device="cuda").manual_seed(sum(sq))
    sk = sk or sq
    q = torch.randn((H, sum(sq), D), generator=g, device="cuda").to(dtype)
    k, v = (torch.randn((H, sum(sk), D), generator=g, device="cuda").to(dtype) for _ in range(2))
    lam = torch.randn(H, generator=g, device="cuda")
    cu_q, cu_k = (torch.tensor([0, *s], device="cuda").cumsum(0).to(torch.int32) for s in (sq, sk))
    o, parts, lse = mg.moga_diff_attn_fwd(q, k, v, lam, cu_q, cu_k, 0.125)
    again, none, lse2 = mg.moga_diff_attn_fwd(q, k, v, lam, cu_q, cu_k, 0.125, want_parts=False)
    assert none is None and torch.equal(again, o) and torch.equal(lse2, lse)
    # O = O_1 - lambda O_2 of the written sums, rounded once in 32 bits
    want = torch.addcmul(parts[0].double(), -lam[:, None, None].double(), parts[1].double()).float().to(dtype)
    assert torch.equal(o, want)
