"""Positions in differential attention: each of a head's two maps is an attention by itself, so its queries and keys are turned within its own
D / 2 channels, and its scores depend on differences of positions alone."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import moga_diff_attention, rotary

from . import block_ref as ref

CASES = [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 128)]


def turn_maps(x, pos, freq, axis_pairs, interleaved, factor=1.0):
    """x [N, H, D] in 64 bits, each half of a head turned as complex numbers.  freq of up to D / 4 pairs: both halves alike; of D / 2: the first half's,
    then the second's.  pos [axes, N]."""
    N, H, D = x.shape
    h, P = D // 2, freq.numel()
    axis = torch.repeat_interleave(torch.arange(pos.shape[0], device=x.device), torch.tensor(axis_pairs, device=x.device))
    angle = pos.double()[axis].t() * freq                        # [N, P]
    maps = []
    for m in range(2):
        part = x[..., m * h:(m + 1) * h]
        a = angle if P <= h // 2 else angle[:, m * (P // 2):(m + 1) * (P // 2)]
        n = a.shape[1]
        z = torch.polar(torch.full_like(a, factor), a)[:, None]
        if interleaved:
            w = torch.view_as_complex(part[..., :2 * n].reshape(N, H, n, 2).contiguous()) * z
            y = torch.view_as_real(w).flatten(2)
        else:
            w = torch.complex(part[..., :n], part[..., n:2 * n]) * z
            y = torch.cat([w.real, w.imag], 2)
        maps.append(torch.cat([y, part[..., 2 * n:]], 2))
    return torch.cat(maps, 2)


def _positions(N, axes):
    i = torch.arange(N)
    return (i[None] if axes == 1 else torch.stack([i // 35, i // 7 % 5, i % 7])).to(torch.int32)


def _dims(total, axes):
    """Channels of each axis, all even."""
    each = total // axes // 2 * 2
    return [total - (axes - 1) * each] + [each] * (axes - 1)


@pytest.mark.parametrize("inter", [False, True])
def test_only_turning_within_a_map_keeps_its_scores(inter):
    """64 bits, the plain forms: a constant added to all positions changes no score of a map turned within itself; turned as one head of D channels in
    halves, it does."""
    D, N = 16, 6
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn((N, 1, D), generator=g, dtype=torch.float64) for _ in range(2))
    score = lambda t, a, b: t(q, a)[:, 0, :D // 2] @ t(k, b)[:, 0, :D // 2].t()
    pos = torch.arange(N, dtype=torch.int32)[None]
    for pairs in (D // 4, D // 2):
        freq = 100.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
        own = lambda x, p: turn_maps(x, p, freq, [pairs], inter)
        assert torch.allclose(score(own, pos, pos), score(own, pos + 50, pos + 50), rtol=1e-10, atol=1e-10)
    freq = 100.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    whole = lambda x, p: ref.rotate(x, p, freq, [D // 2], inter, 1.0)
    same = torch.allclose(score(whole, pos, pos), score(whole, pos + 50, pos + 50), rtol=1e-10, atol=1e-10)
    assert same == inter
    if inter:   # neighbours of the whole head: every pair lies in one map, the first map has the first half of the frequencies
        assert torch.allclose(whole(q, pos), turn_maps(q, pos, freq, [D // 2], True), rtol=1e-12, atol=1e-12)


def test_refusals_of_the_rotation_in_maps():
    import ctypes
    fake, odd, out = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0x2000)
    pairs = lambda *n: (ctypes.c_int * len(n))(*n)
    for name in ("moga_rotary_permute_maps_fwd", "moga_rotary_permute_maps_bwd"):
        c = lambda q=fake, v=fake, dt=1, N=4, H=2, D=128, perm=fake, pos=fake, axes=1, ax=None, f=fake, R=64, each=0, factor=1.0, vo=out: (
            getattr(mg.load(), name)(q, fake, v, dt, N, H, D, perm, pos, axes, ax, f, R, each, 0, factor, out, out, vo, None))
        assert c(N=0) == 0 and c(N=0, q=None) == 0
        assert c(q=None) == -1 and c(v=None) == -1 and c(perm=None) == -1 and c(pos=None) == -1 and c(f=None) == -1 and c(vo=None) == -1
        assert c(N=-1) == -1 and c(H=0) == -1 and c(D=0) == -1
        assert c(R=66) == -1 and c(R=128) == -1 and c(R=7) == -1 and c(R=0) == -1      # channels of a map
        assert c(D=120, R=8) == -2 and c(D=272, R=8) == -2 and c(dt=2) == -2           # a map is a multiple of 8 channels
        assert c(axes=2) == -1 and c(axes=2, ax=pairs(16, 15)) == -1
        assert c(axes=2, ax=pairs(16, 16), each=1) == -1 and c(axes=2, ax=pairs(40, 23), each=1) == -1   # of both maps: 64 pairs
        assert c(q=odd) == -1 and c(vo=fake) == -1 and c(factor=float("nan")) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("share", [2, 1])
@pytest.mark.parametrize("dtype,D", CASES)
def test_output_and_gradients(dtype, D, share, inter, axes):
    """moga_diff_attention with positions against 64 bits: frequencies of one map (D / 2 channels) or of both (D)."""
    N, H, M = 260, 2, 3
    g = torch.Generator().manual_seed(D + axes)
    rnd = lambda *s: torch.randn(s, generator=g)
    t = {n: rnd(N, H, D).to(dtype).cuda().requires_grad_(n != "do") for n in ("q", "k", "v", "do")}
    lam = (rnd(H) * 0.3 + 0.5).cuda().requires_grad_()
    x, w = rnd(N, 32).to(dtype).cuda(), rnd(M, 32).cuda()
    dims = _dims(D // share, axes)
    freq, _ = mg.moga_rotary_freqs(dims, base=100.0)
    pairs, pos, scale = [d // 2 for d in dims], _positions(N, axes).cuda(), (D // 2) ** -0.5
    o, _, group = moga_diff_attention(x, w, t["q"], t["k"], t["v"], lam, scale, positions=pos, inv_freq=freq, axis_pairs=pairs, interleaved=inter,
                                      factor=1.1)
    wrt = [t["q"], t["k"], t["v"], lam]
    got = torch.autograd.grad(o, wrt, t["do"])

    e = [a.detach().double().requires_grad_() for a in wrt]
    gate = torch.softmax(x.double() @ w.double().t(), 1).gather(1, group[:, None].long())
    qr, kr = (turn_maps(a, pos, freq, pairs, inter, 1.1) for a in e[:2])
    ro = torch.zeros((N, H, D), dtype=torch.float64, device="cuda")
    rows = 0.0
    for m in range(M):
        i = (group == m).nonzero()[:, 0]
        if i.numel():
            r = [0, i.numel()]
            part, parts, _ = ref.diff_fwd(*(a[i].transpose(0, 1) for a in (qr, kr, e[2])), e[3], r, r, scale)
            ro = ro.index_add(0, i, part.transpose(0, 1) * gate[i][:, None])
            rows = rows + (gate[i] * (t["do"][i].double() * parts[1].detach().transpose(0, 1)).sum(2)).square().sum(0)
    want = torch.autograd.grad(ro, e, t["do"].double())
    # fp32: some hundred u (2^-24).  bf16: the rotated q and k, the weights, the sorted and the scattered output are rounded one after the other, and as
    # many gradients: ten roundings of 0.0017 rms, 0.0054; a gradient is a difference of two larger parts (dP and delta): up to three times that
    most = 1e-4 if dtype == torch.float32 else 1.6e-2
    ref.near(o, ro, most, "o")
    for n, a, b in zip("dq dk dv".split(), got, want):
        ref.near(a, b, most, n)
    # lambda's gradient is minus the sum of the rows' dO . O_2, of either sign: each row's error is relative to the row, so that the sum's is relative
    # to the root of the rows' squares, not to what is left of them.  (The rounded q, k and dO put into the formula in 64 bits give -2.0322 and
    # 12.9618 where the unrounded ones give -2.1089 and 12.7236, bf16, neighbours, three axes: rows' roots 34.1 and 32.9, 0.005 of them.)
    assert ((got[3].double() - want[3]).abs() <= most * rows.sqrt()).all(), (got[3], want[3], rows.sqrt())


@pytest.mark.gpu
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("share", [2, 1])
def test_a_constant_added_to_all_positions_changes_nothing(share, inter, axes):
    """fp32.  A rotated value is off by at most 10 u (|x1| + |x2|) (test_gpu_rotary.py), a score by what that makes of its products and by the sums of
    block_ref.diff_all; the weights by twice the worst score's error; both results are off."""
    N, H, D, M = 200, 2, 64, 2
    g = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=g).cuda()
    q, k, v, x, w, lam = rnd(N, H, D), rnd(N, H, D), rnd(N, H, D), rnd(N, 16), rnd(M, 16), rnd(H) * 0.3
    dims = _dims(D // share, axes)
    freq, _ = mg.moga_rotary_freqs(dims, base=100.0)
    pairs, pos, scale = [d // 2 for d in dims], _positions(N, axes).cuda(), 0.18
    run = lambda p: moga_diff_attention(x, w, q, k, v, lam, scale, positions=p, inv_freq=freq, axis_pairs=pairs, interleaved=inter)
    a, _, group = run(pos)
    b, _, _ = run(pos + 1000)
    sizes = lambda t: torch.cat([ref.pair_sizes(m, 2 * min(freq.numel(), D // 4), inter) for m in t.double().split(D // 2, 2)], 2)
    bound = torch.zeros((N, H, D), dtype=torch.float64, device="cuda")
    for m in range(M):
        i = (group == m).nonzero()[:, 0]
        Q, K, V = (t[i].double().transpose(0, 1) for t in (q, k, v))
        worst = 0.0
        for s in (slice(0, D // 2), slice(D // 2, D)):
            ts = scale * sizes(q)[i].transpose(0, 1)[..., s] @ sizes(k)[i].transpose(0, 1)[..., s].transpose(1, 2)
            worst = max(worst, float(ts.max()))
        rel = 2 * ref.U * (20 * worst + 0.5 * D // 2 * worst + 8 * worst + 64)
        # weights sum to one: the size of the output's parts is at most that of V
        bound[i] = (2 * rel * (1 + lam.abs())[:, None, None] * V.abs().amax(1, keepdim=True)).expand(-1, i.numel(), -1).transpose(0, 1)
    assert float(bound.max()) < 1e-2   # what is wrong is off by some 0.1
    ref.within(a, b.double(), bound, "o")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("N,H,D,R", [(1, 1, 128, 64), (517, 3, 128, 64), (50, 3, 128, 60), (33, 2, 64, 32), (40, 5, 64, 6), (23, 1, 16, 8), (77, 2, 256, 128),
                                     (20, 2, 48, 22), (4099, 12, 128, 48)])
def test_sorted_order_has_the_bits_of_single_maps(N, H, D, R, inter, dtype):
    """The rotation in maps on the way into the groups is that of 2 H heads of D / 2 channels in token order and the gather."""
    rnd = lambda s: torch.randn((N, H, D), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").to(dtype)
    q, k, v = rnd(1), rnd(2), rnd(3)
    dims = [R] if R < 12 else _dims(R, 3)
    freq, _ = mg.moga_rotary_freqs(dims)
    pos = torch.randint(-900, 90000, (len(dims), N), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    perm = torch.randperm(N, generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    how = dict(axis_pairs=[d // 2 for d in dims], interleaved=inter, factor=1.25)
    half = lambda t: t.view(N, 2 * H, D // 2)
    yq, yk = (y.view(N, H, D) for y in mg.moga_rotary_fwd(half(q), half(k), pos, freq, **how))
    assert all(torch.equal(a, b) for a, b in zip(mg.moga_rotary_fwd(q, k, pos, freq, maps=2, **how), (yq, yk)))
    got = mg.moga_rotary_permute_fwd(q, k, v, perm, pos, freq, maps=2, **how)
    for t, y in zip(got, (yq, yk, v)):
        assert torch.equal(t, y[perm.long()].transpose(0, 1))
    back = mg.moga_rotary_permute_bwd(*got, perm, pos, freq, maps=2, **how)
    tok = [torch.empty_like(q).index_copy_(0, perm.long(), t.transpose(0, 1).contiguous()) for t in got]
    dq, dk = (y.view(N, H, D) for y in mg.moga_rotary_bwd(half(tok[0]), half(tok[1]), pos, freq, **how))
    assert torch.equal(back[0], dq) and torch.equal(back[1], dk) and torch.equal(back[2], v)
    assert all(torch.equal(a, b) for a, b in zip(mg.moga_rotary_bwd(tok[0], tok[1], pos, freq, maps=2, **how), (dq, dk)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("N,H,D", [(1, 2, 128), (70, 3, 128), (45, 2, 64), (19, 1, 16), (33, 1, 48)])
def test_each_map_with_its_own_frequencies(N, H, D, inter, dtype):
    """D / 2 pairs: the first D / 4 turn the first map, the others the second; neighbours are then those of the whole head."""
    rnd = lambda s: torch.randn((N, H, D), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").to(dtype)
    q, k, v = rnd(1), rnd(2), rnd(3)
    freq, _ = mg.moga_rotary_freqs(D)
    pos = torch.arange(N, dtype=torch.int32, device="cuda") * 3
    perm = torch.randperm(N, generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    got = mg.moga_rotary_permute_fwd(q, k, v, perm, pos, freq, interleaved=inter, maps=2)
    maps = []
    for m in range(2):
        part = lambda t: t[..., m * (D // 2):(m + 1) * (D // 2)].contiguous()
        maps.append(mg.moga_rotary_fwd(part(q), part(k), pos, freq[m * (D // 4):(m + 1) * (D // 4)].clone(), interleaved=inter))
    yq, yk = (torch.cat(p, 2) for p in zip(*maps))
    for t, y in zip(got, (yq, yk, v)):
        assert torch.equal(t, y[perm.long()].transpose(0, 1))
    if inter:
        assert all(torch.equal(a, b) for a, b in zip(got, mg.moga_rotary_permute_fwd(q, k, v, perm, pos, freq, interleaved=True)))
    back = mg.moga_rotary_permute_bwd(*got, perm, pos, freq, interleaved=inter, maps=2)
    assert torch.equal(back[2], v)
    # turned there and back: three roundings of at most half a step, of values that two of either size make
    for t, y in ((back[0], q), (back[1], k)):
        r = torch.cat([ref.pair_sizes(p, D // 2, inter) for p in y.double().split(D // 2, 2)], 2)
        ref.within(t, y.double(), (3 * ref.HALF_STEP[dtype] + 30 * ref.U) * r, "there and back")


@pytest.mark.gpu
def test_autograd_of_the_rotation_in_maps():
    N, H, D = 70, 2, 64
    rnd = lambda s: torch.randn((N, H, D), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda")
    q, k, dq, dk = rnd(1), rnd(2), rnd(3), rnd(4)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D // 2)
    a, b = q.clone().requires_grad_(True), k.clone().requires_grad_(True)
    y = rotary(a, b, pos, freq, maps=2)
    assert all(torch.equal(s, t) for s, t in zip(y, mg.moga_rotary_fwd(q, k, pos, freq, maps=2)))
    got = torch.autograd.grad(y, [a, b], [dq, dk])
    assert all(torch.equal(s, t) for s, t in zip(got, mg.moga_rotary_bwd(dq, dk, pos, freq, maps=2)))


@pytest.mark.gpu
def test_refuses_frequencies_that_fit_no_map():
    N, H, D = 10, 2, 64
    q = torch.randn((N, H, D), device="cuda")
    pos, perm = torch.arange(N, dtype=torch.int32, device="cuda"), torch.arange(N, dtype=torch.int32, device="cuda")
    x, w, lam = torch.randn((N, 8), device="cuda"), torch.randn((2, 8), device="cuda"), torch.ones(H, device="cuda")
    for dims in (D // 2 + 2, D - 2):   # more than a map has, fewer than both
        freq, _ = mg.moga_rotary_freqs(dims)
        with pytest.raises(ValueError):
            moga_diff_attention(x, w, q, q, q, lam, 0.1, positions=pos, inv_freq=freq)
        with pytest.raises(ValueError):
            mg.moga_rotary_permute_fwd(q, q, q, perm, pos, freq, maps=2)
    with pytest.raises(ValueError):
        mg.moga_rotary_fwd(q, q, pos, mg.moga_rotary_freqs(D)[0], maps=2)
    for maps in (0, 3):
        with pytest.raises(ValueError):
            mg.moga_rotary_fwd(q, q, pos, mg.moga_rotary_freqs(16)[0], maps=maps)
        with pytest.raises(ValueError):
            mg.moga_rotary_permute_fwd(q, q, q, perm, pos, mg.moga_rotary_freqs(16)[0], maps=maps)
