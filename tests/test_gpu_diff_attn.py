"""Differential attention, forward and backward, against 64 bits; the bounds are block_ref.diff_all's."""
import ctypes

import pytest
import torch

from paper_2510_18692_amd import binding as mg

from . import block_ref as ref

pytestmark = pytest.mark.gpu

# rms of a rounding to bf16 is 2^-8 / sqrt(3) / 1.4 = 0.0017 of the value; an output sums rounded weights and is rounded itself: 0.0024, and a third
# more for the sums of two maps
NEAR = {torch.bfloat16: 3.5e-3, torch.float32: 5e-6}


def _cu(sizes):
    out = [0]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def _inputs(H, D, dtype, cu_q, cu_k, seed, spread=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randn((H, n, D), generator=g, device="cuda")
    q, k, v, do = rnd(cu_q[-1]).to(dtype), (rnd(cu_k[-1]) * spread).to(dtype), rnd(cu_k[-1]).to(dtype), rnd(cu_q[-1]).to(dtype)
    lam = torch.rand(H, generator=g, device="cuda") * 2 - 0.8
    return q, k, v, do, lam


def _dev(cu):
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def _run(q, k, v, do, lam, cu_q, cu_k, scale):
    o, parts, lse = mg.moga_diff_attn_fwd(q, k, v, lam, _dev(cu_q), _dev(cu_k), scale)
    dq, dk, dv, dlam = mg.moga_diff_attn_bwd(do, q, k, v, parts, lse, lam, _dev(cu_q), _dev(cu_k), scale)
    return dict(o=o, parts=parts, lse=lse, dq=dq, dk=dk, dv=dv, dlam=dlam)


def _check(got, q, k, v, do, lam, cu_q, cu_k, scale, near=True):
    want = ref.diff_all(q.double(), k.double(), v.double(), lam.double(), do.double(), cu_q, cu_k, scale, ref.HALF_STEP[q.dtype])
    for name, (r, bound) in want.items():
        if name == "lse":
            assert torch.equal(got[name] == -torch.inf, r == -torch.inf)
            r, bound, t = r.nan_to_num(neginf=0.0), bound, got[name].nan_to_num(neginf=0.0)
            ref.within(t, r, bound, name)
            continue
        ref.within(got[name], r, bound, name)
        if near and name in ("o", "dq", "dk", "dv"):
            ref.near(got[name], r, NEAR[q.dtype], name)


SHAPES = {   # queries and keys of each group
    "one": ([1], [1]),
    "single queries": ([1] * 5, [1, 2, 33, 700, 31]),
    "edges": ([15, 16, 17, 31, 32, 33], [33, 32, 31, 17, 16, 15]),
    "tiles": ([63, 64, 65, 127, 128, 129], [129, 128, 127, 65, 64, 63]),
    "none on one side": ([0, 40, 0, 70, 0, 5], [30, 0, 0, 90, 1, 0]),
    "long keys": ([40, 3], [1500, 2200]),
    "long queries": ([1300, 700], [20, 90]),
    "equal": ([300, 0, 1, 450, 77, 128], None),
}


@pytest.mark.parametrize("H,D,dtype", [(3, 128, torch.bfloat16), (2, 128, torch.float32), (3, 64, torch.float32)])
@pytest.mark.parametrize("name", SHAPES)
def test_against_64_bits(name, H, D, dtype):
    sq, sk = SHAPES[name]
    cu_q, cu_k = _cu(sq), _cu(sk or sq)
    t = _inputs(H, D, dtype, cu_q, cu_k, len(name) + D)
    scale = (D // 2) ** -0.5
    _check(_run(*t, cu_q, cu_k, scale), *t, cu_q, cu_k, scale, near=name not in ("one", "single queries"))   # there gradients cancel


@pytest.mark.parametrize("H,D,dtype", [(17, 128, torch.bfloat16), (9, 64, torch.float32)])
def test_more_heads_than_xcds(H, D, dtype):
    cu = _cu([100, 230, 0, 64])
    t = _inputs(H, D, dtype, cu, cu, 4)
    _check(_run(*t, cu, cu, 0.125), *t, cu, cu, 0.125)


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_more_groups_than_the_lookup_takes(D, dtype):
    sizes = [(7 * i) % 23 for i in range(400)]
    keys = [(5 * i + 3) % 41 for i in range(400)]
    cu_q, cu_k = _cu(sizes), _cu(keys)
    t = _inputs(2, D, dtype, cu_q, cu_k, 6)
    _check(_run(*t, cu_q, cu_k, 0.125), *t, cu_q, cu_k, 0.125, near=False)


@pytest.mark.parametrize("groups,longest", [(5, 3000), (70, 700), (300, 200)])
def test_a_few_queries_a_group(groups, longest):
    """Groups of 0 to 40 queries, 8 on average, and 0 to `longest` keys."""
    g = torch.Generator().manual_seed(groups)
    cu_q = _cu([int(x) for x in torch.randint(0, 17, (groups - 1,), generator=g)] + [40])
    cu_k = _cu([longest] + [int(x) for x in torch.randint(0, longest + 1, (groups - 1,), generator=g)])
    t = _inputs(2, 128, torch.bfloat16, cu_q, cu_k, 31)
    _check(_run(*t, cu_q, cu_k, 0.125), *t, cu_q, cu_k, 0.125, near=False)


@pytest.mark.parametrize("spread", [1e-3, 12.0, 60.0])
@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (128, torch.float32)])
def test_flat_and_peaked_maps(D, dtype, spread):
    cu = _cu([200, 333])
    t = _inputs(2, D, dtype, cu, cu, 8, spread)
    _check(_run(*t, cu, cu, 0.125), *t, cu, cu, 0.125, near=spread < 1 or dtype == torch.float32 and spread < 20)


def test_rising_scores_move_the_maximum():
    """Keys in ascending order of their scores: the running maximum is raised again and again, by much and by little."""
    n, D = 600, 128
    q = torch.zeros((1, 40, D), device="cuda")
    q[..., 0] = q[..., 64] = 1.0
    k = torch.zeros((1, n, D), device="cuda")
    k[0, :, 0] = torch.arange(n, device="cuda") * 0.5
    k[0, :, 64] = torch.arange(n, device="cuda") * -0.5
    v = torch.randn((1, n, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    do, lam = torch.randn_like(q), torch.tensor([0.5], device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        t = (q.to(dtype), k.to(dtype), v.to(dtype), do.to(dtype), lam)
        _check(_run(*t, [0, 40], [0, n], 1.0), *t, [0, 40], [0, n], 1.0, near=False)


@pytest.mark.parametrize("H,D,dtype", [(2, 128, torch.bfloat16), (2, 64, torch.float32), (1, 128, torch.float32)])
@pytest.mark.parametrize("sq,sk", [([1, 1, 1], [5000, 300, 9000]), ([3], [4000]), ([1, 0, 2], [3000, 3000, 0]), ([130], [2600]), ([1, 1], [6000, 1])])
def test_split_keys(sq, sk, H, D, dtype):
    """Few queries: with room the keys are split over the chip, without it they are not; either is right, and both give every output."""
    cu_q, cu_k = _cu(sq), _cu(sk)
    q, k, v, do, lam = _inputs(H, D, dtype, cu_q, cu_k, 5)
    code = {torch.float32: 0, torch.bfloat16: 1}[dtype]
    need = mg.workspace_bytes(mg.OP_DIFF_ATTN_FWD, cu_q[-1], H, D, len(sq), 0, code)
    room = mg.load().moga_workspace_preferred_bytes(mg.OP_DIFF_ATTN_FWD, cu_q[-1], cu_k[-1], H, D, len(sq), 0, code)
    assert room > need
    want = ref.diff_all(q.double(), k.double(), v.double(), lam.double(), do.double(), cu_q, cu_k, 0.1, ref.HALF_STEP[dtype])
    dcq, dck = _dev(cu_q), _dev(cu_k)
    for size in (need, room):
        o, parts, lse = torch.empty_like(q), torch.empty((2, *q.shape), device="cuda"), torch.empty((2, *q.shape[:2]), device="cuda")
        ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device="cuda")
        p = lambda x: ctypes.c_void_p(x.data_ptr())
        st = mg.load().moga_diff_attn_fwd(p(q), p(k), p(v), code, cu_q[-1], cu_k[-1], H, D, p(lam), p(dcq), p(dck), len(sq), 0.1, p(o), p(parts),
                                          p(lse), p(ws), size, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0
        for name, t in (("o", o), ("parts", parts)):
            ref.within(t, *want[name], f"{name}, {size} bytes")
        assert torch.equal(lse == -torch.inf, want["lse"][0] == -torch.inf)
        ref.within(lse.nan_to_num(neginf=0.0), want["lse"][0].nan_to_num(neginf=0.0), want["lse"][1], "lse")


@pytest.mark.parametrize("H,D,dtype", [(2, 128, torch.bfloat16), (2, 64, torch.float32), (1, 128, torch.float32)])
@pytest.mark.parametrize("sq,sk", [([700], [900]), ([1500, 3], [2, 1100]), ([40, 0, 1300], [2000, 300, 0]), ([1], [3000]), ([2600], [1])])
def test_split_backward(sq, sk, H, D, dtype):
    """Few tiles: with room either sweep is shared out over the chip, without it neither is; bits repeat with as much room."""
    cu_q, cu_k = _cu(sq), _cu(sk)
    q, k, v, do, lam = _inputs(H, D, dtype, cu_q, cu_k, 25)
    code, Nq, Nk, G = {torch.float32: 0, torch.bfloat16: 1}[dtype], cu_q[-1], cu_k[-1], len(sq)
    need = mg.workspace_bytes(mg.OP_DIFF_ATTN_BWD, Nq, H, D, G, 0, code)
    room = mg.load().moga_workspace_preferred_bytes(mg.OP_DIFF_ATTN_BWD, Nq, Nk, H, D, G, 0, code)
    assert room > need
    want = ref.diff_all(q.double(), k.double(), v.double(), lam.double(), do.double(), cu_q, cu_k, 0.1, ref.HALF_STEP[dtype])
    dcq, dck = _dev(cu_q), _dev(cu_k)
    _, parts, lse = mg.moga_diff_attn_fwd(q, k, v, lam, dcq, dck, 0.1)
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    for size in (need, room):
        seen = []
        for _ in range(2):
            out = {"dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v), "dlam": torch.empty_like(lam)}
            ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
            st = mg.load().moga_diff_attn_bwd(p(do), p(q), p(k), p(v), p(parts), p(lse), code, Nq, Nk, H, D, p(lam), p(dcq), p(dck), G, 0.1,
                                              *(p(out[n]) for n in ("dq", "dk", "dv", "dlam")), p(ws), size,
                                              ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
            assert st == 0
            for name, t in out.items():
                ref.within(t, *want[name], f"{name}, {size} bytes")
            seen.append(out)
        assert all(torch.equal(seen[0][n], seen[1][n]) for n in seen[0])


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_other_groups_values_never_leak(D, dtype):
    """Infinities and NaN in one group's rows: the other groups keep their bits."""
    cu_q, cu_k = _cu([40, 33, 70]), _cu([45, 10, 100])
    q, k, v, do, lam = _inputs(2, D, dtype, cu_q, cu_k, 21)
    a = _run(q, k, v, do, lam, cu_q, cu_k, 0.125)
    q, k, v, do = (x.clone() for x in (q, k, v, do))
    q[:, 40:73], do[:, 45:50], k[:, 45:55], v[:, 45:50], v[:, 50] = float("nan"), float("inf"), float("-inf"), float("nan"), float("inf")
    b = _run(q, k, v, do, lam, cu_q, cu_k, 0.125)
    for name, rows in (("o", cu_q), ("dq", cu_q), ("dk", cu_k), ("dv", cu_k)):
        for g in (0, 2):
            assert torch.equal(a[name][:, rows[g]:rows[g + 1]], b[name][:, rows[g]:rows[g + 1]]), (name, g)
    assert b["o"][:, 40:73].isnan().all()


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_rows_behind_the_last_group_stay(D, dtype):
    H, code = 2, {torch.float32: 0, torch.bfloat16: 1}[dtype]
    cu_q, cu_k = _cu([50, 61]), _cu([64, 33])
    q, k, v, do, lam = _inputs(H, D, dtype, [0, 140], [0, 130], 2)
    want = ref.diff_all(*(x[:, :cu_q[-1]].double() if i in (0, 3) else x[:, :cu_k[-1]].double() if i < 3 else x.double()
                          for i, x in ((0, q), (1, k), (2, v), (4, lam), (3, do))), cu_q, cu_k, 0.125, ref.HALF_STEP[dtype])
    new = lambda n, **kw: torch.full((H, n, D), 5.0, device="cuda", dtype=dtype)
    o, dq, dk, dv = new(140), new(140), new(130), new(130)
    parts, lse, dlam = torch.full((2, H, 140, D), 5.0, device="cuda"), torch.full((2, H, 140), 5.0, device="cuda"), torch.empty(H, device="cuda")
    dcq, dck = _dev(cu_q), _dev(cu_k)
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    lib = mg.load()
    for size in (mg.workspace_bytes(mg.OP_DIFF_ATTN_FWD, 140, H, D, 2, 0, code),
                 lib.moga_workspace_preferred_bytes(mg.OP_DIFF_ATTN_FWD, 140, 130, H, D, 2, 0, code)):
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        assert lib.moga_diff_attn_fwd(p(q), p(k), p(v), code, 140, 130, H, D, p(lam), p(dcq), p(dck), 2, 0.125, p(o), p(parts), p(lse), p(ws), size, st) == 0
        ref.within(o[:, :111], *want["o"], "o")
        assert (o[:, 111:] == 5).all() and (parts[:, :, 111:] == 5).all() and (lse[:, :, 111:] == 5).all()
    size = mg.workspace_bytes(mg.OP_DIFF_ATTN_BWD, 140, H, D, 2, 0, code)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    assert lib.moga_diff_attn_bwd(p(do), p(q), p(k), p(v), p(parts), p(lse), code, 140, 130, H, D, p(lam), p(dcq), p(dck), 2, 0.125, p(dq), p(dk), p(dv),
                                  p(dlam), p(ws), size, st) == 0
    for name, t, n in (("dq", dq, 111), ("dk", dk, 97), ("dv", dv, 97)):
        ref.within(t[:, :n], *want[name], name)
        assert (t[:, n:] == 5).all(), name
    ref.within(dlam, *want["dlam"], "dlam")


@pytest.mark.parametrize("n", [12, 70, 250])
def test_gradients_of_short_groups(n):
    """Two roundings to bf16 lie between the formulas and dQ or dK: dS as an operand and the result, sqrt(2) of the result's own.  The operand's is not
    centred as dS is: keys drawn towards a query, (spread^2 scale)^2 64 of spread^2 64 = 3.5 % more, sqrt(2.035) = 1.427; 2 % for a finite sum."""
    H, G = 12, max(3, 1500 // n)
    cu = _cu([n] * G)
    q, k, v, do, lam = _inputs(H, 128, torch.bfloat16, cu, cu, n)
    got = _run(q, k, v, do, lam, cu, cu, 0.125)
    want = ref.diff_all(q.double(), k.double(), v.double(), lam.double(), do.double(), cu, cu, 0.125, ref.HALF_STEP[q.dtype])
    for name in ("dq", "dk"):
        r = want[name][0]
        own = (r.bfloat16().double() - r).norm()
        assert (got[name].double() - r).norm() <= 1.455 * own, name


def test_gradient_of_lambda_over_many_rows():
    """60,000 rows whose parts have either sign: errors of single rows average out, a common one adds up.  An eighth of u a row, common to all, is
    60,000 u / 8 of a sum of some 0.4 sqrt(60,000): 4.6e-6."""
    H, D, n, G = 3, 128, 5000, 12
    cu = _cu([n] * G)
    q, k, v, do, lam = _inputs(H, D, torch.bfloat16, cu, cu, 77)
    got = _run(q, k, v, do, lam, cu, cu, 0.125)["dlam"]
    want = torch.zeros(H, dtype=torch.float64, device="cuda")
    for g in range(G):
        r = slice(cu[g], cu[g + 1])
        for h in range(H):
            p = torch.softmax(0.125 * q[h, r, 64:].double() @ k[h, r, 64:].double().t(), 1)
            want[h] -= (p * (do[h, r].double() @ v[h, r].double().t())).sum()
    ref.near(got, want, 4.6e-6, "dlam")


def test_repeated_calls_give_the_same_bits():
    cu = _cu([500, 120, 900])
    t = _inputs(4, 128, torch.bfloat16, cu, cu, 17)
    a = _run(*t, cu, cu, 0.125)
    for _ in range(3):
        b = _run(*t, cu, cu, 0.125)
        assert all(torch.equal(a[n], b[n]) for n in a)


def test_keys_without_queries_leave_the_rows_behind_them():
    k = torch.randn((2, 9, 128), device="cuda").bfloat16()
    dk, dv, dlam = torch.full_like(k, 5), torch.full_like(k, 5), torch.full((2,), 5.0, device="cuda")
    lam, cq, ck = torch.ones(2, device="cuda"), _dev([0, 0]), _dev([0, 6])
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    st = mg.load().moga_diff_attn_bwd(None, None, p(k), p(k), None, None, 1, 0, 9, 2, 128, p(lam), p(cq), p(ck), 1, 0.1, None, p(dk), p(dv), p(dlam), None,
                                      0, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert st == 0 and (dlam == 0).all()
    for t in (dk, dv):
        assert (t[:, :6] == 0).all() and (t[:, 6:] == 5).all()


def test_nothing_on_a_side():
    lam = torch.ones(2, device="cuda")
    e, k = torch.empty((2, 0, 128), device="cuda", dtype=torch.bfloat16), torch.randn((2, 9, 128), device="cuda").bfloat16()
    r = _run(e, k, k, e, lam, [0, 0], [0, 9], 0.1)
    assert (r["dk"] == 0).all() and (r["dv"] == 0).all() and (r["dlam"] == 0).all()
    r = _run(k, e, e, k, lam, [0, 9], [0, 0], 0.1)
    assert (r["o"] == 0).all() and (r["dq"] == 0).all() and (r["lse"] == -torch.inf).all() and (r["dlam"] == 0).all()


def test_refuses_tensors_that_do_not_fit():
    q = torch.randn((2, 8, 128), device="cuda").bfloat16()
    lam, cu = torch.ones(2, device="cuda"), _dev([0, 8])
    ok = (q, q, q, lam, cu, cu, 0.1)
    o, parts, lse = mg.moga_diff_attn_fwd(*ok)
    for i, bad, kind in ((1, q.float(), TypeError), (2, q[:, :4].contiguous(), ValueError), (3, lam[:1], ValueError), (3, lam.double(), TypeError),
                         (4, cu.long(), TypeError), (5, _dev([0, 4, 8]), ValueError), (0, q[0], ValueError), (1, q.transpose(0, 1), AssertionError)):
        args = list(ok)
        args[i] = bad
        with pytest.raises(kind):
            mg.moga_diff_attn_fwd(*args)
    with pytest.raises(mg.MogaError):
        mg.moga_diff_attn_fwd(q, q, q, lam, cu, cu, -0.1)
    with pytest.raises(mg.MogaError):   # bf16 heads are 128 wide
        h = q[..., :64].contiguous()
        mg.moga_diff_attn_fwd(h, h, h, lam, cu, cu, 0.1)
    with pytest.raises(TypeError):
        mg.moga_diff_attn_bwd(q, q, q, q, parts.bfloat16(), lse, lam, cu, cu, 0.1)
    with pytest.raises(ValueError):
        mg.moga_diff_attn_bwd(q, q, q, q, parts[0].contiguous(), lse, lam, cu, cu, 0.1)
