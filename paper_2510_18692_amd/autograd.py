"""torch.autograd wrappers around the C-ABI calls (argument marshalling only).

    o, lb = moga_attention(x, w, q, k, v, scale, balance_alpha=0.1)

`o` is the output of Alg. 1 with the gate of Eq. 5, `lb` the group balancing loss of Eqs. 6-8 (or
None).  Gradients flow to q, k, v and to the router weight w (through the gate, and through the
balancing loss when it is used); the assignment itself is a constant of differentiation.  No
gradient is returned for the router input x unless `grad_x=True` (the optional dX of the router
backward).  Everything runs in the HIP library; the autograd function itself is native
(csrc/torch_binding.cpp), so that the backward pass does not enter the interpreter.
`layer_norm`, `residual_norm`, `gated_ffn`, `rotary` and `moga_diff_attention` have first derivatives only: gradients taken with
create_graph=True raise an error where they are differentiated again.  Before a step whose backward is captured into a graph, let go of the eager
results of the same leaves (see moga_diff_attention).
"""
from __future__ import annotations

from . import binding as mg


def moga_attention(x, w, q, k, v, softmax_scale, balance_alpha=None, grad_x=False):
    """x [N, d_model], w [M, d_model] fp32, q/k/v [N, H, D] -> (o [N, H, D], balancing loss or None, group [N])."""
    o, loss, group = mg._nat.attention(x, w, q, k, v, softmax_scale, balance_alpha, grad_x)
    return o, (loss if balance_alpha is not None else None), group


def layer_norm(x, weight=None, bias=None, eps=1e-6):
    """Layer norm over the last axis of x [..., C] (contiguous), weight and bias f32 [C] or None -> y like x."""
    return mg._nat.layer_norm(x, weight, bias, eps)


def residual_norm(x, y=None, gate=None, post_weight=None, weight=None, bias=None, scale=None, shift=None, post="none", pre="layer", residual_scale=1.0,
                  tokens_per_row=None, eps=1e-6, dtype=None):
    """r = x + residual_scale * gate * post(y) * post_weight, and h = (pre(r) * weight + bias) * (1 + scale) + shift, in one pass
    (binding.moga_residual_norm_fwd): x, y [..., C] (contiguous) -> (r, which is x without y; h, None without pre)."""
    return mg._nat.residual_norm(x, y, gate, post_weight, weight, bias, scale, shift, mg._one_of(mg.NORMS, post, "post"),
                                 mg._one_of(mg.NORMS, pre, "pre"), residual_scale, tokens_per_row, eps, dtype)


def gated_ffn(x, w_in, w_out, activation="silu"):
    """(act(a) * u) w_out^T with [a, u] = x w_in^T: x [..., C] (contiguous), w_in [2 F, C], w_out [C, F] (binding.moga_gated_ffn_fwd) -> y like x."""
    return mg._nat.gated_ffn(x, w_in, w_out, mg._one_of(mg.ACTIVATIONS, activation, "activation"))


def rotary(q, k, positions, inv_freq, axis_pairs=None, interleaved=False, factor=1.0, maps=1):
    """Rotary positions of q [N, Hq, D] and k [N, Hk, D], either may be None (binding.moga_rotary_fwd; maps=2 before moga_diff_attention) -> (qo, ko)."""
    return mg._nat.rotary_apply(q, k, positions, inv_freq, axis_pairs or [], interleaved, factor, maps)


def moga_diff_attention(x, w, q, k, v, lam, softmax_scale, balance_alpha=None, grad_x=False, positions=None, inv_freq=None, axis_pairs=None,
                        interleaved=False, factor=1.0):
    """moga_attention with differential attention in the groups: the two halves of a head's channels are two maps, lam f32 [H] the weight of
    the second (moga_diff_attn_fwd); gradients flow to lam as well.  With positions and inv_freq q and k are rotated on their way into the groups, each map
    within its own D / 2 channels: inv_freq of at most D / 4 pairs (binding.moga_rotary_freqs(D // 2)) turns both maps alike, one of D / 2 pairs has the
    first map's and then the second's (binding.moga_rotary_permute_fwd, maps=2).  -> (o [N, H, D], balancing loss or None, group [N]).
    A step whose backward is captured into a graph: let go of the eager results of the same leaves before the capture (torch keeps the stream
    on which a leaf was first used, and a capture may not join work of another)."""
    o, loss, group = mg._nat.diff_attention(x, w, q, k, v, lam, softmax_scale, balance_alpha, grad_x, positions, inv_freq, axis_pairs or [],
                                            interleaved, factor)
    return o, (loss if balance_alpha is not None else None), group
