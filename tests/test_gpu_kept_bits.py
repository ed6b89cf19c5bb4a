"""What the feed-forward's backward makes of the kept a and u, to one rounding."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg

from .test_gpu_gated_ffn import _inputs
from .test_gpu_gated_ffn_tiles import tiles   # noqa: F401
from .test_kept_bits import off, parts

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("how", [None, (0, 1, 1), (0, 1000, 3), (1, 1, 1), (1, 1000, 2), (2, 1, 1), (2, 1000, 2)])
@pytest.mark.parametrize("N", [5, 300])
def test_kept_bits_reach_the_gradients(tiles, N, how, act):
    """With d_y = W_out = 1 in one channel and 0 elsewhere dh is 1, and with W_in one each [da, du] are d_x: from the a and u that the forward kept, to one
    rounding.  N = 5: kept by the kernel of few tokens."""
    F, C = 264, 528
    x, wi, wo, _ = _inputs(N, C, F, BF, 6)
    _, au, h = mg.moga_gated_ffn_fwd(x, wi, wo, act)
    dy, one = torch.zeros_like(x), torch.zeros_like(wo)
    dy[:, 0], one[0] = 1, 1
    if how:
        tiles(*how)
    d_x, _, _ = mg.moga_gated_ffn_bwd(dy, x, torch.eye(2 * F, device="cuda", dtype=BF), one, au, h, act, want_dw_in=False, want_dw_out=False)
    assert off(d_x, *parts(au, N, F), act) <= 1
