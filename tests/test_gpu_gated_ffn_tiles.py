"""Every kernel that the feed-forward's products can take, at small sizes, against 64 bits."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg

from .test_gpu_gated_ffn import _check

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def tiles():
    yield mg.set_ffn_tiles
    mg.set_ffn_tiles()


# (tiles to a round, splits): all of them whole, all split in two and in more (the last run of k shorter), whole rounds of two or three with a split rest
CUTS = [(1, 1), (1000, 2), (1000, 3), (2, 4), (3, 2)]


@pytest.mark.parametrize("round,splits", CUTS)
@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("N,C,F", [(300, 264, 520), (257, 776, 264), (1090, 72, 136), (600, 512, 256)])
def test_bf16(tiles, N, C, F, shape, round, splits):
    for together, act in ((True, "silu"), (False, "gelu")):
        tiles(shape, round, splits, together)
        _check(N, C, F, BF, act)


@pytest.mark.parametrize("round,splits", CUTS)
@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("N,C,F", [(300, 132, 260), (150, 388, 132), (530, 36, 68), (256, 256, 128)])
def test_f32(tiles, N, C, F, shape, round, splits):
    for together, act in ((True, "gelu"), (False, "gelu_tanh")):
        tiles(shape, round, splits, together)
        _check(N, C, F, F32, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype,N,C,F", [(F32, 33, 36, 68), (F32, 48, 132, 260), (F32, 49, 512, 1368), (F32, 64, 100, 1028), (F32, 20, 1028, 36), (BF, 49, 264, 520)])
def test_few_tokens(dtype, N, C, F, act):
    _check(N, C, F, dtype, act)


def test_the_calls_choose_again(tiles):
    size = lambda: mg.workspace_bytes(mg.OP_GATED_FFN_BWD, 300, 0, 520, 1, 264, 1)
    own = size()
    tiles(0, 1, 1)
    whole = size()
    tiles(0, 1000, 3)
    assert size() > whole
    tiles()
    assert size() == own
