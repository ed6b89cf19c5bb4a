"""The operators together, as a layer uses them: layer norm of the hidden state, the projections, layer norm of queries and keys by head, rotary
positions on the way into the groups, differential attention inside them, the gated scatter -- and the gradients of all of it."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg
from paper_2510_18692_amd.autograd import layer_norm, moga_diff_attention, rotary

from . import block_ref as ref

pytestmark = pytest.mark.gpu


def _layer64(p, scale, pairs, freq, pos, group, alpha):
    """The layer in 64 bits by torch's autograd, the assignment given."""
    N, H, D = p["do"].shape
    M = p["w"].shape[0]
    norm = lambda t, w, b: ref.norm_fwd(t, w, b, 1e-5)[0]
    h = norm(p["x"], p["nw"], p["nb"])
    q, k, v = ((h @ p[n]).view(N, H, D) for n in ("wq", "wk", "wv"))
    q, k = norm(q, p["qw"], None), norm(k, None, None)
    q, k = (ref.rotate(t, pos, freq, pairs, True, 1.0) for t in (q, k))
    prob = torch.softmax(h @ p["w"].t(), 1)
    gate = prob.gather(1, group[:, None].long())
    o = torch.zeros((N, H, D), dtype=torch.float64, device="cuda")
    loss = 0.0
    for g in range(M):
        i = (group == g).nonzero()[:, 0]
        frac = i.numel() / N
        loss = loss + alpha * M * frac * gate[i].sum() / N
        if i.numel():
            part, _, _ = ref.diff_fwd(*(t[i].transpose(0, 1) for t in (q, k, v)), p["lam"], [0, i.numel()], [0, i.numel()], scale)
            o = o.index_add(0, i, part.transpose(0, 1) * gate[i][:, None])
    return o, loss


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 128)])
def test_layer(dtype, D, fused):
    N, H, M, dm = 333, 2, 5, 96
    g = torch.Generator().manual_seed(D)
    rnd = lambda *s: torch.randn(s, generator=g)
    p = {"x": rnd(N, dm), "nw": rnd(dm) * 0.2 + 1, "nb": rnd(dm) * 0.1, "wq": rnd(dm, H * D) * dm ** -0.5, "wk": rnd(dm, H * D) * dm ** -0.5,
         "wv": rnd(dm, H * D) * dm ** -0.5, "qw": rnd(D) * 0.2 + 1, "w": rnd(M, dm) * dm ** -0.5, "lam": rnd(H) * 0.3 + 0.5, "do": rnd(N, H, D)}
    keep = {"nw", "nb", "qw", "w", "lam"}   # fp32 beside bf16 tensors
    leaves = {n: t.to(torch.float32 if n in keep else dtype).cuda().requires_grad_(n != "do") for n, t in p.items()}
    pos = torch.stack([torch.arange(N) // 60, torch.arange(N) // 10 % 6, torch.arange(N) % 10]).to(torch.int32).cuda()
    dims = [D - 2 * (D // 6 * 2), D // 6 * 2, D // 6 * 2]
    freq, _ = mg.moga_rotary_freqs(dims)
    pairs, scale = [d // 2 for d in dims], (D // 2) ** -0.5

    def layer(t):
        h = layer_norm(t["x"], t["nw"], t["nb"], 1e-5)
        q, k, v = ((h @ t[n]).view(N, H, D) for n in ("wq", "wk", "wv"))
        q, k = layer_norm(q, t["qw"], None, 1e-5), layer_norm(k, None, None, 1e-5)
        if fused:
            return moga_diff_attention(h, t["w"], q, k, v, t["lam"], scale, 0.1, True, pos, freq, pairs, True)
        q, k = rotary(q, k, pos, freq, pairs, True)
        return moga_diff_attention(h, t["w"], q, k, v, t["lam"], scale, 0.1, True)

    o, loss, group = layer(leaves)
    wrt = [n for n in leaves if n != "do"]
    grads = torch.autograd.grad([o, loss], [leaves[n] for n in wrt], [leaves["do"], torch.ones_like(loss)])
    exact = {n: t.detach().double().requires_grad_(n != "do") for n, t in leaves.items()}
    ro, rl = _layer64(exact, scale, pairs, freq, pos, group, 0.1)
    rg = torch.autograd.grad([ro, rl], [exact[n] for n in wrt], [exact["do"], torch.ones_like(rl)])
    # fp32: some hundred u through seven operators.  bf16: ten tensors are rounded one after the other (0.0017 rms each, 0.0017 sqrt(10) = 0.0054), and
    # gradients pass as many again: 0.0076; gradients of x and the projections are differences of two larger parts (norm's means): twice that
    most = 1e-4 if dtype == torch.float32 else 1.6e-2
    ref.near(o, ro, most, "o")
    ref.near(loss, rl, most, "loss")
    for n, a, b in zip(wrt, grads, rg):
        ref.near(a, b, most, n)


def test_forward_and_backward_in_a_graph_match_eager_on_every_replay():
    N, H, D, M = 700, 3, 128, 4
    rnd = lambda s, *shape: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").bfloat16()
    x, dy = rnd(1, N, 256), rnd(2, N, 256)
    w = torch.ones(256, device="cuda") * 1.5
    q, k, v, do = (rnd(i, N, H, D) for i in (3, 4, 5, 6))
    lam = torch.full((H,), 0.4, device="cuda")
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D)
    group = torch.randint(0, M, (N,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    one_q, cu1 = rnd(9, H, 2, D), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    long_k, cuk = rnd(10, H, 5000, D), torch.tensor([0, 4000, 5000], dtype=torch.int32, device="cuda")

    def run():
        y, mean, rstd = mg.moga_layer_norm_fwd(x, w, w)
        out = [y, *mg.moga_layer_norm_bwd(dy, x, w, mean, rstd), *mg.moga_rotary_fwd(q, k, pos, freq), *mg.moga_rotary_bwd(q, k, pos, freq)]
        pm = mg.moga_permute(group, M)
        qh, kh, vh = mg.moga_rotary_permute_fwd(q, k, v, pm["perm"], pos, freq)
        oh, parts, lse = mg.moga_diff_attn_fwd(qh, kh, vh, lam, pm["cu_seqlens"], pm["cu_seqlens"], 0.125)
        d = mg.moga_diff_attn_bwd(mg.moga_gather_rows(do, pm["perm"]), qh, kh, vh, parts, lse, lam, pm["cu_seqlens"], pm["cu_seqlens"], 0.125)
        out += [oh, lse, *d, *mg.moga_rotary_permute_bwd(*d[:3], pm["perm"], pos, freq)]
        return out + [mg.moga_diff_attn_fwd(one_q, long_k, long_k, lam, cu1, cuk, 0.125, want_parts=False)[0]]

    eager = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for rep in range(3):
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), rep
        again = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, eager)), rep


def test_captured_training_step():
    """Forward and backward through the autograd functions in one graph, of leaves that no eager graph holds."""
    N, H, D, M = 700, 3, 128, 4
    rnd = lambda s, *shape: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda")
    x, w, g = rnd(1, N, 64).bfloat16(), rnd(2, M, 64), rnd(6, N, H, D).bfloat16()
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D)

    def leaves():
        t = [w, rnd(3, N, H, D).bfloat16(), rnd(4, N, H, D).bfloat16(), rnd(5, N, H, D).bfloat16(), torch.full((H,), 0.3, device="cuda"),
             torch.ones(D, device="cuda")]
        return [a.clone().requires_grad_() for a in t]

    def step(t):
        q = layer_norm(t[1], t[5])
        o, loss, _ = moga_diff_attention(x, t[0], q, t[2], t[3], t[4], 0.125, balance_alpha=0.1, positions=pos, inv_freq=freq)
        return [o.detach(), *torch.autograd.grad([o, loss], t, [g, torch.ones_like(loss)])]

    want = [a.clone() for a in step(leaves())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(leaves())
    torch.cuda.synchronize()
    own = leaves()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(own)
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), rep
        again = step(leaves())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), rep
        del again


def test_on_another_stream():
    """Given a stream that is not the current one: inputs made there, outputs in its order, temporaries not reused too early."""
    side = torch.cuda.Stream()
    H, D = 4, 128
    rnd = lambda s, *shape: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").bfloat16()
    q, do = rnd(1, H, 900, D), rnd(2, H, 900, D)
    lam, cu = torch.full((H,), 0.3, device="cuda"), torch.tensor([0, 400, 900], dtype=torch.int32, device="cuda")
    x, w = rnd(3, 900, 512), torch.ones(512, device="cuda")
    pos = torch.arange(900, dtype=torch.int32, device="cuda")
    freq, _ = mg.moga_rotary_freqs(D)
    t = q.transpose(0, 1).contiguous()

    def run(**kw):
        o, parts, lse = mg.moga_diff_attn_fwd(q, q, q, lam, cu, cu, 0.125, **kw)
        d = mg.moga_diff_attn_bwd(do, q, q, q, parts, lse, lam, cu, cu, 0.125, **kw)
        y, mean, rstd = mg.moga_layer_norm_fwd(x, w, w, **kw)
        n = mg.moga_layer_norm_bwd(x, x, w, mean, rstd, **kw)
        return [o, *d, y, *n, *mg.moga_rotary_fwd(t, t, pos, freq, **kw)]

    want = run()
    torch.cuda.synchronize()
    for _ in range(3):
        got = run(stream=side)
        noise = [torch.full((900, 512), 7.0, device="cuda") for _ in range(20)]   # would take memory that is given back too early
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del noise


def test_two_calls_at_once():
    """Two streams, each with calls of its own workspaces."""
    H, D = 4, 128
    rnd = lambda s: torch.randn((H, 1500, D), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").bfloat16()
    a, b = rnd(1), rnd(2)
    lam, cu = torch.full((H,), 0.3, device="cuda"), torch.tensor([0, 600, 1500], dtype=torch.int32, device="cuda")

    def run(t):
        o, parts, lse = mg.moga_diff_attn_fwd(t, t, t, lam, cu, cu, 0.125)
        return [o, *mg.moga_diff_attn_bwd(t, t, t, t, parts, lse, lam, cu, cu, 0.125)]

    want = run(a), run(b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s1):
            x = run(a)
        with torch.cuda.stream(s2):
            y = run(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(x, want[0])) and all(torch.equal(p, q) for p, q in zip(y, want[1]))


def test_no_tokens():
    e = lambda *s: torch.empty(s, device="cuda", requires_grad=True)
    lam = torch.full((2,), 0.3, device="cuda", requires_grad=True)
    q, k, v = e(0, 2, 64), e(0, 2, 64), e(0, 2, 64)
    o, loss, _ = moga_diff_attention(torch.empty((0, 32), device="cuda"), torch.randn((3, 32), device="cuda"), q, k, v, lam, 0.125)
    assert o.shape == (0, 2, 64)
    grads = torch.autograd.grad(o, [q, k, v, lam], torch.empty_like(o))
    assert all(g.shape == t.shape for g, t in zip(grads, (q, k, v, lam))) and (grads[3] == 0).all()
    y = layer_norm(torch.empty((0, 3, 16), device="cuda", requires_grad=True))
    assert y.shape == (0, 3, 16)


def test_unrouted_gradients_and_no_grad():
    N, H, D = 64, 2, 64
    rnd = lambda s, *shape: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda")
    x, w, q = rnd(1, N, 32), rnd(2, 3, 32), rnd(3, N, H, D)
    lam = torch.full((H,), 0.3, device="cuda", requires_grad=True)
    o, loss, group = moga_diff_attention(x, w, q, q, q, lam, 0.125)
    assert loss is None and group.dtype == torch.int32 and not group.requires_grad
    o.sum().backward()
    assert lam.grad.shape == (H,) and lam.grad.isfinite().all()
    with torch.no_grad():
        again, _, _ = moga_diff_attention(x, w, q, q, q, lam, 0.125)
    assert torch.equal(again, o) and not again.requires_grad
    with pytest.raises(ValueError):
        moga_diff_attention(x, w, q, q, q, lam[:1].detach(), 0.125)
    with pytest.raises(ValueError):
        moga_diff_attention(x, w, q, q, q, lam, 0.125, positions=torch.arange(N, dtype=torch.int32).cuda())
