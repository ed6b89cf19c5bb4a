"""Layer norm, rotary positions and differential attention without a GPU: the tests' own formulas against difference quotients, the host
builder of the angles, workspace sizes, and every refusal."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2510_18692_amd import binding as mg

from . import block_ref as ref

FAKE = ctypes.c_void_p(0x1000)   # aligned, never read: the checks come first
ODD = ctypes.c_void_p(0x1004)


def _quotients(f, x, i, h=1e-6):
    """Central differences of f's scalar result by the entries i of x."""
    out = []
    for j in i:
        y = x.clone().view(-1)
        y[j] += h
        a = f(y.view(x.shape))
        y[j] -= 2 * h
        out.append(float((a - f(y.view(x.shape))) / (2 * h)))
    return out


def test_reference_gradients_are_difference_quotients():
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, w, b, dy = rnd(5, 7), rnd(7), rnd(7), rnd(5, 7)
    dx, dw, db = ref.norm_bwd(dy, x, w, 1e-3)
    f = lambda x, w, b: (ref.norm_fwd(x, w, b, 1e-3)[0] * dy).sum()
    assert np.allclose(_quotients(lambda t: f(t, w, b), x, range(35)), dx.view(-1), rtol=1e-6, atol=1e-7)
    assert np.allclose(_quotients(lambda t: f(x, t, b), w, range(7)), dw, rtol=1e-6, atol=1e-7)
    assert np.allclose(_quotients(lambda t: f(x, w, t), b, range(7)), db, rtol=1e-6, atol=1e-7)

    x, d = rnd(6, 2, 8), rnd(6, 2, 8)
    pos, freq = torch.arange(6)[None] * 7 - 9, torch.tensor([1.0, 0.3, 0.01], dtype=torch.float64)
    for inter in (False, True):
        back = ref.rotate(d, pos, freq, [3], inter, 1.3, -1)
        got = _quotients(lambda t: (ref.rotate(t, pos, freq, [3], inter, 1.3) * d).sum(), x, range(96))
        assert np.allclose(got, back.view(-1), rtol=1e-6, atol=1e-7)

    H, D, cu_q, cu_k = 2, 8, [0, 3, 3, 4, 6], [0, 2, 5, 9, 9]
    q, k, v, do, lam = rnd(H, 6, D), rnd(H, 9, D), rnd(H, 9, D), rnd(H, 6, D), torch.tensor([0.7, -0.4], dtype=torch.float64)
    r = ref.diff_all(q, k, v, lam, do, cu_q, cu_k, 0.5, ref.U)
    f = lambda q, k, v, lam: (ref.diff_fwd(q, k, v, lam, cu_q, cu_k, 0.5)[0] * do).sum()
    assert np.allclose(_quotients(lambda t: f(t, k, v, lam), q, range(q.numel())), r["dq"][0].view(-1), rtol=1e-5, atol=1e-7)
    assert np.allclose(_quotients(lambda t: f(q, t, v, lam), k, range(k.numel())), r["dk"][0].view(-1), rtol=1e-5, atol=1e-7)
    assert np.allclose(_quotients(lambda t: f(q, k, t, lam), v, range(v.numel())), r["dv"][0].view(-1), rtol=1e-5, atol=1e-7)
    assert np.allclose(_quotients(lambda t: f(q, k, v, t), lam, range(2)), r["dlam"][0], rtol=1e-5, atol=1e-7)
    assert (r["o"][0][:, 4:] == 0).all() and torch.isinf(r["lse"][0][:, :, 4:]).all()


def test_reference_of_one_map_is_plain_attention():
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((1, 9, 8), generator=g, dtype=torch.float64) for _ in range(3))
    o, _, lse = ref.diff_fwd(q, k, v, torch.zeros(1, dtype=torch.float64), [0, 9], [0, 9], 0.5)
    p = torch.softmax(0.5 * q[..., :4] @ k[..., :4].transpose(1, 2), 2)
    assert torch.allclose(o, p @ v, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("R", [2, 6, 128])
def test_angles(R):
    n = R // 2
    base = np.array([10000.0 ** (-i / n) for i in range(n)])
    got, factor = mg.moga_rotary_freqs(R, device="cpu")
    assert got.dtype == torch.float64 and factor == 1.0
    assert np.allclose(got.numpy(), base, rtol=1e-14)
    got, factor = mg.moga_rotary_freqs(R, scaling="linear", scale_factor=4.0, device="cpu")
    assert factor == 1.0 and np.allclose(got.numpy(), base / 4, rtol=1e-14)
    got, factor = mg.moga_rotary_freqs(R, scaling="base", scale_factor=4.0, device="cpu")
    assert factor == 1.0 and got[0] == 1.0
    if n > 1:   # the slowest pair is slowed down by the factor
        assert math.isclose(float(got[-1]), base[-1] / 4, rel_tol=1e-12)
    got, factor = mg.moga_rotary_freqs(R, scaling="parts", scale_factor=4.0, original_len=4096, device="cpu")
    assert math.isclose(factor, 0.1 * math.log(4) + 1, rel_tol=1e-6)
    turns = 4096 * base / (2 * math.pi)
    for f, b, t in zip(got.numpy(), base, turns):
        assert math.isclose(f, b if t >= 32 else b / 4 if t <= 1 else b * ((t - 1) / 31) + b / 4 * (1 - (t - 1) / 31), rel_tol=1e-12)


def test_angles_of_axes_lie_one_after_the_other():
    got, _ = mg.moga_rotary_freqs([44, 42, 42], base=500.0, device="cpu")
    assert got.shape == (64,)
    assert torch.equal(got[:22], mg.moga_rotary_freqs(44, base=500.0, device="cpu")[0])
    assert torch.equal(got[22:43], got[43:])
    assert mg.moga_rotary_freqs([4, 0], device="cpu")[0].shape == (2,)   # an axis without pairs


def test_angle_builder_refuses():
    f = (ctypes.c_double * 64)()
    x = ctypes.c_float()
    call = lambda R=8, base=1e4, kind=0, s=1.0, n=0.0, fast=32.0, slow=1.0, out=f, factor=ctypes.byref(x): mg.load().moga_rotary_build_freqs(
        R, base, kind, s, n, fast, slow, out, factor)
    assert call() == 0
    assert call(R=-2) == -1 and call(R=7) == -1 and call(base=0.0) == -1 and call(base=float("nan")) == -1 and call(base=float("inf")) == -1
    assert call(out=None) == -1 and call(factor=None) == -1
    assert call(kind=4) == -2 and call(kind=-1) == -2
    assert call(kind=1, s=0.5) == -1 and call(kind=2, s=float("nan")) == -1
    assert call(kind=3, s=2.0) == -1 and call(kind=3, s=2.0, n=100.0) == 0
    assert call(kind=3, s=2.0, n=100.0, fast=1.0) == -1 and call(kind=3, s=2.0, n=100.0, slow=0.0) == -1
    with pytest.raises(ValueError):
        mg.moga_rotary_freqs(8, scaling="other", device="cpu")
    with pytest.raises(mg.MogaError):
        mg.moga_rotary_freqs(7, device="cpu")


def test_layer_norm_refuses():
    fwd = lambda x=FAKE, dt=1, w=FAKE, b=FAKE, N=4, C=64, eps=1e-6, y=FAKE, m=FAKE, r=FAKE: mg.load().moga_layer_norm_fwd(
        x, dt, w, b, N, C, eps, y, m, r, None)
    assert fwd(N=0) == 0 and fwd(N=0, x=None, y=None) == 0
    assert fwd(x=None) == -1 and fwd(y=None) == -1 and fwd(m=None) == -1 and fwd(r=None) == -1
    assert fwd(N=-1) == -1 and fwd(C=0) == -1 and fwd(C=-8) == -1
    assert fwd(eps=-1.0) == -1 and fwd(eps=float("nan")) == -1 and fwd(eps=float("inf")) == -1
    assert fwd(dt=2) == -2 and fwd(C=16385) == -2 and fwd(N=1 << 31) == -2
    assert fwd(x=ODD) == -1 and fwd(y=ODD) == -1 and fwd(w=ODD) == -1 and fwd(b=ODD) == -1
    ws = mg.workspace_bytes(mg.OP_LAYER_NORM_BWD, 4, 0, 0, 1, 64, 1)
    assert ws >= 2 * 64 * 4
    bwd = lambda dy=FAKE, x=FAKE, dt=1, w=FAKE, m=FAKE, r=FAKE, N=4, C=64, dx=FAKE, dw=FAKE, db=FAKE, p=FAKE, n=ws: (
        mg.load().moga_layer_norm_bwd(dy, x, dt, w, m, r, N, C, dx, dw, db, p, n, None))
    assert bwd(dy=None) == -1 and bwd(x=None) == -1 and bwd(m=None) == -1 and bwd(r=None) == -1 and bwd(dx=None) == -1
    assert bwd(N=-1) == -1 and bwd(C=0) == -1 and bwd(dt=7) == -2 and bwd(C=20000) == -2
    assert bwd(dx=ODD) == -1 and bwd(dw=ODD) == -1 and bwd(p=ODD) == -1
    assert bwd(p=None) == -3 and bwd(n=ws - 1) == -3 and bwd(dw=None, n=0) == -3
    assert bwd(N=0, dw=None, db=None, p=None, n=0) == 0


def test_layer_norm_workspace():
    wb = lambda N, C, dt: mg.workspace_bytes(mg.OP_LAYER_NORM_BWD, N, 0, 0, 1, C, dt)
    assert wb(0, 64, 1) == 0 and wb(10, 0, 1) == 0 and wb(10, 64, 9) == 0
    sizes = [wb(N, 5120, 1) for N in (1, 10, 1000, 100000, 10000000)]
    assert sizes == sorted(sizes) and sizes[-1] <= 64 << 20


def test_rotary_refuses():
    pairs = lambda *n: (ctypes.c_int * len(n))(*n)
    out = ctypes.c_void_p(0x2000)

    def call(name, q=FAKE, k=FAKE, dt=1, N=4, Hq=2, Hk=2, D=128, pos=FAKE, axes=1, ax=None, f=FAKE, R=128, factor=1.0, qo=out, ko=out):
        return getattr(mg.load(), name)(q, k, dt, N, Hq, Hk, D, pos, axes, ax, f, R, 0, factor, qo, ko, None)

    for name in ("moga_rotary_fwd", "moga_rotary_bwd"):
        assert call(name, N=0) == 0 and call(name, N=0, q=None) == 0
        assert call(name, q=None) == -1 and call(name, ko=None) == -1 and call(name, pos=None) == -1 and call(name, f=None) == -1
        assert call(name, N=-1) == -1 and call(name, Hq=-1) == -1 and call(name, Hq=0, Hk=0) == -1 and call(name, D=0) == -1
        assert call(name, R=0) == -1 and call(name, R=7) == -1 and call(name, R=130) == -1
        assert call(name, factor=float("nan")) == -1 and call(name, factor=float("inf")) == -1
        assert call(name, dt=3) == -2 and call(name, D=132, R=4) == -2 and call(name, D=264, R=4) == -2 and call(name, N=1 << 28) == -2
        assert call(name, axes=0) == -1 and call(name, axes=5, ax=pairs(60, 1, 1, 1, 1)) == -2
        assert call(name, axes=3) == -1 and call(name, axes=3, ax=pairs(22, 21, 20)) == -1 and call(name, axes=2, ax=pairs(65, -1)) == -1
        assert call(name, qo=FAKE) == -1   # in place
        assert call(name, q=ODD) == -1 and call(name, ko=ODD) == -1 and call(name, pos=ODD) == -1
    for name in ("moga_rotary_permute_fwd", "moga_rotary_permute_bwd"):
        c = lambda q=FAKE, v=FAKE, H=2, perm=FAKE, R=128, vo=out: getattr(mg.load(), name)(
            q, FAKE, v, 1, 4, H, 128, perm, FAKE, 1, None, FAKE, R, 0, 1.0, out, out, vo, None)
        assert c(q=None) == -1 and c(v=None) == -1 and c(perm=None) == -1 and c(vo=None) == -1 and c(H=0) == -1 and c(R=200) == -1


def test_differential_attention_refuses():
    def fwd(q=FAKE, k=FAKE, v=FAKE, dt=1, Nq=8, Nk=8, H=2, D=128, lam=FAKE, cq=FAKE, ck=FAKE, G=2, scale=0.1, o=FAKE, parts=None, lse=FAKE, ws=None, n=0):
        return mg.load().moga_diff_attn_fwd(q, k, v, dt, Nq, Nk, H, D, lam, cq, ck, G, scale, o, parts, lse, ws, n, None)

    assert fwd(Nq=0) == 0 and fwd(Nq=0, q=None, o=None) == 0
    for name in ("q", "k", "v", "lam", "cq", "ck", "o", "lse"):
        assert fwd(**{name: None}) == -1, name
    for name in ("q", "k", "v", "o", "parts", "ws"):
        assert fwd(**{name: ODD}) == -1, name
    assert fwd(Nq=-1) == -1 and fwd(Nk=-1) == -1 and fwd(H=0) == -1 and fwd(G=0) == -1 and fwd(D=0) == -1
    assert fwd(scale=0.0) == -1 and fwd(scale=float("nan")) == -1 and fwd(scale=-1.0) == -1 and fwd(scale=float("inf")) == -1
    assert fwd(dt=2) == -2 and fwd(D=64) == -2 and fwd(dt=0, D=96) == -2 and fwd(Nq=1 << 24) == -2 and fwd(dt=0, Nk=1 << 24) == -2
    assert fwd(G=(1 << 24) + 1) == -2
    assert fwd(G=300) == -3 and fwd(G=300, ws=FAKE, n=300 * 4) == -3
    assert mg.workspace_bytes(mg.OP_DIFF_ATTN_FWD, 8, 2, 128, 256, 0, 1) == 0
    assert mg.workspace_bytes(mg.OP_DIFF_ATTN_FWD, 8, 2, 128, 300, 0, 1) >= 301 * 4

    need = mg.workspace_bytes(mg.OP_DIFF_ATTN_BWD, 8, 2, 128, 2, 0, 1)

    def bwd(do=FAKE, q=FAKE, k=FAKE, v=FAKE, parts=FAKE, lse=FAKE, dt=1, Nq=8, Nk=8, H=2, D=128, lam=FAKE, cq=FAKE, ck=FAKE, G=2, scale=0.1, dq=FAKE,
            dk=FAKE, dv=FAKE, dl=FAKE, ws=FAKE, n=need):
        return mg.load().moga_diff_attn_bwd(do, q, k, v, parts, lse, dt, Nq, Nk, H, D, lam, cq, ck, G, scale, dq, dk, dv, dl, ws, n, None)

    for name in ("do", "q", "k", "v", "parts", "lse", "lam", "cq", "ck", "dq", "dk", "dv", "dl"):
        assert bwd(**{name: None}) == -1, name
    for name in ("do", "q", "k", "v", "parts", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: ODD}) == -1, name
    assert bwd(ws=None) == -3 and bwd(n=need - 1) == -3
    assert bwd(dt=5) == -2 and bwd(D=64) == -2 and bwd(scale=0.0) == -1 and bwd(G=0) == -1 and bwd(H=0) == -1


def test_pieces_need_room_only_where_tiles_are_few():
    pref = lambda Nq, Nk, H, G, dt=1: mg.load().moga_workspace_preferred_bytes(mg.OP_DIFF_ATTN_FWD, Nq, Nk, H, 128, G, 0, dt)
    assert pref(4, 4 * 16384, 12, 4) > 0          # one query in each of four groups
    assert pref(99840, 99840, 40, 16) == 0
    assert pref(4, 4 * 100, 12, 4) == 0           # too few keys to share out
    assert pref(0, 100000, 12, 4) == 0


def test_pieces_of_many_heads_and_long_lists_fit_their_types():
    """Room grows with what is split, never past a gigabyte, and no product of sizes wraps."""
    for Nq, Nk, H, G in ((1, (1 << 24) - 1, 60000, 1), (16, (1 << 24) - 1, 4000, 1), (1 << 20, 1 << 23, 64, 1 << 16), ((1 << 24) - 1, 4096, 1, 1),
                         (3000, (1 << 24) - 1, 1, 300)):
        for op in (mg.OP_DIFF_ATTN_FWD, mg.OP_DIFF_ATTN_BWD):
            need = mg.workspace_bytes(op, Nq, H, 128, G, 0, 1)
            room = mg.load().moga_workspace_preferred_bytes(op, Nq, Nk, H, 128, G, 0, 1)
            assert need <= room <= need + (1 << 30), (Nq, Nk, H, G, op)
