"""The gradients of layer norm's weight and bias over many rows, where a row, or a block's share of them, left out or taken twice would show.

Relative distance of the whole gradient from 64 bits.  A column's sum of N products of either sign is some sqrt(N).  fp32 roundings, u = 2^-24, each of rms
u / sqrt(3) of the partial sum: N in the lanes, of sums of 8 to 64 rows (sqrt(8) on average and up), then of sums that grow to the whole one in
16 + 16 + 8 steps at most: sqrt(8 + 40) u / sqrt(3) = 4 u of the result.  xh itself is off by some 3 u of every product, and rows are independent: 3 u more.
5 u = 3e-7; four times that."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg

from . import block_ref as ref

pytestmark = pytest.mark.gpu
MOST = 1.2e-6


# rows to 16 lanes, to a wave and to a block; more than 256 blocks in each, up to the most there are
@pytest.mark.parametrize("N,C", [(70001, 128), (300007, 64), (9000, 512), (140001, 1000), (4500, 1536), (40003, 1535), (2500, 5120), (2301, 8193)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_share_is_lost(N, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(N)
    x, dy = ((torch.randn((N, C), generator=g, device="cuda") * s).to(dtype) for s in (1.5, 1.0))
    w = torch.randn(C, generator=g, device="cuda") + 1
    _, mean, rstd = mg.moga_layer_norm_fwd(x, w, None, 1e-6)
    blocks = mg.workspace_bytes(mg.OP_LAYER_NORM_BWD, N, 0, 0, 1, C, 1 if dtype == torch.bfloat16 else 0) // (8 * C)
    assert blocks > 256   # the second kernel's loop over the blocks runs again
    _, dw, db = mg.moga_layer_norm_bwd(dy, x, w, mean, rstd)
    want_w, want_b = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(0, N, 20000):
        d = dy[a:a + 20000].double()
        xh = ref.norm_fwd(x[a:a + 20000].double(), None, None, 1e-6)[3]
        want_w += (d * xh).sum(0)
        want_b += d.sum(0)
    one = dy[:1].double() * ref.norm_fwd(x[:1].double(), None, None, 1e-6)[3]
    assert one.norm() > 100 * MOST * want_w.norm() and dy[0].double().norm() > 100 * MOST * want_b.norm()   # a single row would show
    ref.near(dw, want_w, MOST, "dw")
    ref.near(db, want_b, MOST, "db")
