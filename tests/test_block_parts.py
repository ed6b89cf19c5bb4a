"""Residual norm and gated feed-forward without a GPU: the tests' formulas against autograd's, workspace sizes, and every refusal of the C calls."""
import ctypes

import pytest
import torch

from paper_2510_18692_amd import binding as mg

from . import block_parts_ref as ref

FAKE = 0x1000   # aligned, never read: the checks come first
ODD = 0x1004


class Args(ctypes.Structure):
    """moga_residual_norm"""
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "y", "gate", "post_weight", "weight", "bias", "scale", "shift")] + [
        ("N", ctypes.c_int64), ("tokens_per_row", ctypes.c_int64)] + [(n, ctypes.c_int) for n in ("C", "x_dtype", "y_dtype", "post", "pre")] + [
        ("residual_scale", ctypes.c_float), ("eps", ctypes.c_float)]


def args(**kw):
    a = dict(x=FAKE, y=FAKE, gate=FAKE, post_weight=FAKE, weight=FAKE, bias=FAKE, scale=FAKE, shift=FAKE, N=4, tokens_per_row=2, C=64, x_dtype=1,
             y_dtype=1, post=1, pre=2, residual_scale=1.0, eps=1e-6)
    return Args(**{**a, **kw})


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms"), ("none", "layer"), ("rms", "none"), ("absent", "rms")])
def test_reference_gradients_of_the_residual_norm(post, pre):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    ref.HALF_STEP[torch.float64] = 0.0
    N, C, each = 7, 6, 3
    t = dict(x=rnd(N, C), y=None if post == "absent" else rnd(N, C))
    p = dict(gate=rnd(3, C), post_weight=rnd(C), weight=rnd(C), bias=rnd(C), scale=rnd(3, C), shift=rnd(3, C))
    for k in ("weight", "bias", "scale", "shift") if pre == "none" else ("gate", "post_weight") if post == "absent" else ("post_weight",) if post == "none" else ():
        p[k] = None
    kind = "none" if post == "absent" else post
    d_r, d_h = (None if post == "absent" else rnd(N, C)), (None if pre == "none" else rnd(N, C))
    leaves = {k: v.requires_grad_() for k, v in {**t, **p}.items() if v is not None}
    with torch.enable_grad():
        out = ref.residual_norm(t["x"], t["y"], p, kind, pre, 0.8, each, 1e-2)
        loss = sum((out[k][0] * d).sum() for k, d in (("r", d_r), ("h", d_h)) if d is not None)
    grads = dict(zip(leaves, torch.autograd.grad(loss, list(leaves.values()))))
    with torch.no_grad():
        got = ref.residual_norm(t["x"], t["y"], p, kind, pre, 0.8, each, 1e-2, d_r, d_h)
    for k, v in grads.items():
        assert torch.allclose(got["d_" + k][0], v, rtol=1e-9, atol=1e-10), k


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_reference_gradients_of_the_feed_forward(act):
    g = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    ref.HALF_STEP[torch.float64] = 0.0
    x, wi, wo, dy = rnd(5, 6).requires_grad_(), rnd(8, 6).requires_grad_(), rnd(6, 4).requires_grad_(), rnd(5, 6)
    grads = torch.autograd.grad((ref.gated_ffn(x, wi, wo, act)["y"][0] * dy).sum(), (x, wi, wo))
    with torch.no_grad():
        got = ref.gated_ffn(x, wi, wo, act, dy)
        like = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
                "gelu_tanh": lambda a: torch.nn.functional.gelu(a, approximate="tanh")}[act](x)
        assert torch.allclose(ref.activation(x, act)[0], like)
    for k, v in zip(("d_x", "d_w_in", "d_w_out"), grads):
        assert torch.allclose(got[k][0], v, rtol=1e-9, atol=1e-10), k


def test_residual_norm_refuses():
    fwd = lambda r=FAKE, h=FAKE, st=FAKE, **kw: mg.load().moga_residual_norm_fwd(ctypes.byref(args(**kw)), r, h, st, None)
    assert mg.load().moga_residual_norm_fwd(None, FAKE, FAKE, FAKE, None) == -1
    assert fwd(N=0) == 0 and fwd(N=0, x=None, r=None, h=None) == 0
    assert fwd(x=None) == -1 and fwd(r=None) == -1 and fwd(h=None) == -1
    assert fwd(N=-1) == -1 and fwd(C=0) == -1 and fwd(tokens_per_row=0) == -1 and fwd(tokens_per_row=-3) == -1
    assert fwd(eps=-1.0) == -1 and fwd(eps=float("nan")) == -1 and fwd(eps=float("inf")) == -1
    assert fwd(residual_scale=float("nan")) == -1 and fwd(residual_scale=float("inf")) == -1
    assert fwd(C=16385) == -2 and fwd(N=1 << 31) == -2 and fwd(x_dtype=2) == -2 and fwd(y_dtype=0) == -2 and fwd(y_dtype=3, x_dtype=0) == -2
    assert fwd(post=3) == -2 and fwd(pre=-1) == -2
    assert fwd(post=0) == -1   # with a weight of it
    assert fwd(y=None) == -1 and fwd(y=None, gate=None, post_weight=None) == -1 and fwd(y=None, gate=None, post=0) == -1
    assert fwd(pre=0) == -1 and fwd(pre=0, weight=None, bias=None, scale=None) == -1
    assert fwd(y=None, gate=None, post_weight=None, post=0, pre=0, weight=None, bias=None, scale=None, shift=None) == -1
    for k in ("x", "y", "gate", "post_weight", "weight", "bias", "scale", "shift"):
        assert fwd(**{k: ODD}) == -1, k
    assert fwd(r=ODD) == -1 and fwd(h=ODD) == -1 and fwd(st=ODD) == -1

    ws = mg.workspace_bytes(mg.OP_RESIDUAL_NORM_BWD, 4, 0, 0, 2, 64, 1)
    assert ws >= 2 * 3 * 64 * 4
    names = ("stats", "d_r", "d_h", "d_x", "d_y", "d_gate", "d_post_weight", "d_weight", "d_bias", "d_scale", "d_shift", "p")

    def bwd(n=ws, **kw):
        given = {k: kw.pop(k, FAKE) for k in names}
        return mg.load().moga_residual_norm_bwd(ctypes.byref(args(**kw)), *given.values(), n, None)
    assert bwd(stats=None) == -1 and bwd(d_h=None) == -1 and bwd(d_x=None) == -1 and bwd(d_y=None) == -1 and bwd(x=None) == -1
    for k in names:
        assert bwd(**{k: ODD}) == -1, k
    for k in ("gate", "post_weight", "weight", "bias", "scale", "shift"):
        assert bwd(**{k: None}) == -1, k   # a gradient of what is not there
    assert bwd(p=None) == -3 and bwd(n=ws - 1) == -3
    assert bwd(C=0) == -1 and bwd(N=-1) == -1 and bwd(x_dtype=5) == -2 and bwd(C=20000) == -2
    off = dict.fromkeys(("d_gate", "d_post_weight", "d_weight", "d_bias", "d_scale", "d_shift"))
    assert bwd(N=0, n=0, p=None, **off) == 0


def test_residual_norm_workspace():
    wb = lambda N, M, C: mg.workspace_bytes(mg.OP_RESIDUAL_NORM_BWD, N, 0, 0, M, C, 1)
    assert wb(0, 1, 64) == 0 and wb(10, 0, 64) == 0 and wb(10, 11, 64) == 0 and wb(10, 1, 0) == 0
    sizes = [wb(N, 1, 5120) for N in (1, 10, 1000, 100000, 10000000)]
    assert sizes == sorted(sizes) and sizes[-1] <= 128 << 20
    assert wb(100000, 1000, 5120) > wb(100000, 1, 5120)


@pytest.mark.parametrize("C", [24, 96, 300, 512, 520, 1536, 5120, 16384])
def test_residual_norm_workspace_grows_with_the_tokens(C):
    """Room for the longest call is room for every shorter one, with one row of the gate or rows of as many tokens."""
    wb = lambda N, M: mg.workspace_bytes(mg.OP_RESIDUAL_NORM_BWD, N, 0, 0, M, C, 1)
    for each in (1 << 40, 1000, 97, 1):
        sizes = [wb(N, -(-N // each)) for N in [*range(1, 5000), *range(5000, 300000, 331)]]
        assert sizes == sorted(sizes), each


def test_gated_ffn_refuses():
    fwd = lambda x=FAKE, wi=FAKE, wo=FAKE, dt=1, N=4, C=64, F=32, act=0, h=FAKE, au=FAKE, y=FAKE, p=FAKE, n=1 << 40: mg.load().moga_gated_ffn_fwd(
        x, wi, wo, dt, N, C, F, act, h, au, y, p, n, None)
    assert fwd(N=0) == 0 and fwd(N=0, x=None, wi=None, wo=None, h=None, y=None) == 0
    assert fwd(x=None) == -1 and fwd(wi=None) == -1 and fwd(wo=None) == -1 and fwd(h=None) == -1 and fwd(y=None) == -1
    assert fwd(N=-1) == -1 and fwd(C=0) == -1 and fwd(F=-8) == -1
    assert fwd(dt=2) == -2 and fwd(act=3) == -2 and fwd(act=-1) == -2 and fwd(N=1 << 31) == -2
    assert fwd(C=60) == -2 and fwd(F=36) == -2 and fwd(dt=0, C=62) == -2 and fwd(C=65544) == -2 and fwd(F=262152) == -2
    for k in ("x", "wi", "wo", "h", "au", "y", "p"):
        assert fwd(**{k: ODD}) == -1, k
    need = mg.workspace_bytes(mg.OP_GATED_FFN_FWD, 300, 0, 8192, 1, 128, 1)
    assert need > 0 and fwd(N=300, C=128, F=8192, p=None) == -3 and fwd(N=300, C=128, F=8192, n=need - 1) == -3

    ws = mg.workspace_bytes(mg.OP_GATED_FFN_BWD, 4, 0, 32, 1, 64, 1)
    assert ws >= 4 * 64 * 2
    bwd = lambda dy=FAKE, x=FAKE, wi=FAKE, wo=FAKE, au=FAKE, h=FAKE, dt=1, N=4, C=64, F=32, act=0, dx=FAKE, dwi=FAKE, dwo=FAKE, p=FAKE, n=ws: (
        mg.load().moga_gated_ffn_bwd(dy, x, wi, wo, au, h, dt, N, C, F, act, dx, dwi, dwo, p, n, None))
    assert bwd(dy=None) == -1 and bwd(x=None) == -1 and bwd(wi=None) == -1 and bwd(wo=None) == -1 and bwd(au=None) == -1 and bwd(h=None) == -1
    assert bwd(N=-1) == -1 and bwd(C=0) == -1 and bwd(dt=7) == -2 and bwd(C=68) == -2 and bwd(act=9) == -2
    for k in ("dy", "x", "wi", "wo", "au", "h", "dx", "dwi", "dwo", "p"):
        assert bwd(**{k: ODD}) == -1, k
    assert bwd(p=None) == -3 and bwd(n=ws - 1) == -3
    assert bwd(dx=None, dwi=None, dwo=None, p=None) == 0 and bwd(N=0, dwi=None, dwo=None, p=None) == 0


def test_gated_ffn_takes_what_fits_a_launch():
    """x is not there: -1 for sizes that are taken, -2 for others."""
    fwd = lambda N, C, F, dt: mg.load().moga_gated_ffn_fwd(None, FAKE, FAKE, dt, N, C, F, 0, FAKE, None, FAKE, FAKE, 1 << 40, None)
    bwd = lambda N, C, F, dt: mg.load().moga_gated_ffn_bwd(None, FAKE, FAKE, FAKE, FAKE, FAKE, dt, N, C, F, 0, FAKE, None, None, FAKE, 1 << 60, None)
    for call in (fwd, bwd):
        assert call(4000000, 5120, 13696, 1) == -1 and call(4000000, 5120, 13696, 0) == -1
        for dt, rows, most in ((1, 256, 2 ** 23 - 2 ** 13), (0, 128, 2 ** 24 - 2 ** 14)):
            assert call(rows * (most - 1), 8, 8, dt) == -1 and call(rows * most, 8, 8, dt) == -2
            assert call((1 << 31) - 1, 65536, 8, dt) == -2 and call((1 << 31) - 1, 8, 262144, dt) == -2
        assert call((1 << 31) - 1, 512, 1368, 1) == -2 and call(1, 65536, 262144, 1) == -1
    assert mg.workspace_bytes(mg.OP_GATED_FFN_BWD, 4000000, 0, 13696, 1, 5120, 1) >= 4000000 * 2 * 13696 * 2


def test_gated_ffn_workspace():
    wb = lambda op, N, C, F, dt: mg.workspace_bytes(op, N, 0, F, 1, C, dt)
    for op in (mg.OP_GATED_FFN_FWD, mg.OP_GATED_FFN_BWD):
        assert wb(op, 0, 64, 32, 1) == 0 and wb(op, 10, 60, 32, 1) == 0 and wb(op, 10, 64, 32, 5) == 0
    assert 0 < wb(mg.OP_GATED_FFN_FWD, 1, 5120, 13696, 1) <= 16 * 5120 * 4   # splits of one token's second product
    assert wb(mg.OP_GATED_FFN_FWD, 32760, 1536, 4096, 1) == 0               # whole rounds of tiles
    assert max(wb(mg.OP_GATED_FFN_FWD, n, 1536, 4096, 1) for n in range(1, 3000, 37)) <= 32 * 256 * 65536 * 4
    assert wb(mg.OP_GATED_FFN_BWD, 32760, 1536, 4096, 1) >= 32760 * 8192 * 2


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("C,F", [(8, 8), (128, 8192), (264, 520), (512, 1368), (1536, 4096), (5120, 13696), (72, 4104)])
def test_gated_ffn_room_for_any_number_of_tokens(C, F, dt):
    """The preferred bytes grow with the tokens and are enough for every shorter call."""
    for op in (mg.OP_GATED_FFN_FWD, mg.OP_GATED_FFN_BWD):
        room = lambda N: mg.load().moga_workspace_preferred_bytes(op, N, 0, 0, F, 1, C, dt)
        need, last = 0, 0
        for N in [*range(1, 700), *range(700, 9000, 29), *range(9000, 140000, 1777)]:
            need = max(need, mg.workspace_bytes(op, N, 0, F, 1, C, dt))
            if N < 80 or N % 7 == 0:
                assert need <= room(N) and last <= room(N), (op, N)
                last = room(N)
        assert room(100000) <= room(100001) and room(0) == 0
