"""Differential attention of few queries a group over long lists of keys: more groups than the lookup scans, and more pieces than are put together at
a time."""
import pytest
import torch

from paper_2510_18692_amd import binding as mg

from . import block_ref as ref
from .test_gpu_diff_attn import _check, _cu, _dev, _inputs, _run

BF16 = 1


def _room(cu_q, cu_k, H):
    """(needed, preferred) bytes of a forward call."""
    G = len(cu_q) - 1
    need = mg.workspace_bytes(mg.OP_DIFF_ATTN_FWD, cu_q[-1], H, 128, G, 0, BF16)
    return need, mg.load().moga_workspace_preferred_bytes(mg.OP_DIFF_ATTN_FWD, cu_q[-1], cu_k[-1], H, 128, G, 0, BF16)


def _lists(groups, longest, queries):
    """Some groups with a query or more, most with none; 0 to `longest` keys, and one group with all of them."""
    g = torch.Generator().manual_seed(groups)
    sq = torch.bincount(torch.randint(0, groups, (queries,), generator=g), minlength=groups)
    return _cu(sq.tolist()), _cu([longest] + [int(x) for x in torch.randint(0, longest + 1, (groups - 1,), generator=g)])


MANY = [(257, 600, 3), (300, 600, 64), (1100, 300, 41)]


@pytest.mark.parametrize("groups,longest,queries", MANY)
def test_the_lists_are_split_by_their_keys(groups, longest, queries):
    """Tiles of 128 queries are split from 512 keys of a mean group on: any room beyond the lookup's is that of pieces of keys."""
    cu_q, cu_k = _lists(groups, longest, queries)
    need, room = _room(cu_q, cu_k, 12)
    assert cu_k[-1] < 512 * groups and need >= 4 * (groups + 1) and room > need


@pytest.mark.gpu
@pytest.mark.parametrize("groups,longest,queries", MANY)
def test_more_groups_than_the_lookup_scans(groups, longest, queries):
    cu_q, cu_k = _lists(groups, longest, queries)
    t = _inputs(12, 128, torch.bfloat16, cu_q, cu_k, 33)
    _check(_run(*t, cu_q, cu_k, 0.125), *t, cu_q, cu_k, 0.125, near=False)


# one group has most of the queries
SKEWED = [(12, [1] * 256 + [3800], [1000] * 256 + [3800]), (1, [1] * 399 + [6001], [4000] * 400), (3, [1] * 40 + [300], [400] * 41)]


@pytest.mark.parametrize("H,sq,sk", SKEWED)
def test_many_queries_are_no_few(H, sq, sk):
    """diff_few_kernel reads a group's keys for every 16 queries, and the host does not know the groups: it is taken where all queries in one group would
    be four times that.  By tiles these calls are whole (room for the lookup alone) or in 16 pieces at most."""
    need, room = _room(_cu(sq), _cu(sk), H)
    assert room <= need + 16 * sum(sq) * H * 2 * 130 * 4 and (sum(sq) < 1000 or room == need)


@pytest.mark.gpu
def test_one_long_group_among_single_queries():
    H, sq, sk = SKEWED[2]
    cu_q, cu_k = _cu(sq), _cu(sk)
    t = _inputs(H, 128, torch.bfloat16, cu_q, cu_k, 35)
    _check(_run(*t, cu_q, cu_k, 0.125), *t, cu_q, cu_k, 0.125, near=False)
    cu_q = _cu([1, 1, 61, 1])   # few in all: four times 16 in one group
    cu_k = _cu([700, 300, 900, 1200])
    t = _inputs(H, 128, torch.bfloat16, cu_q, cu_k, 36)
    _check(_run(*t, cu_q, cu_k, 0.125), *t, cu_q, cu_k, 0.125, near=False)


LONG = [([1, 2], [40000, 17000]), ([3, 0, 1], [17000, 400, 66000]), ([16], [20000])]


@pytest.mark.parametrize("sq,sk", LONG)
def test_long_lists_have_more_than_64_pieces(sq, sk):
    cu_q, cu_k = _cu(sq), _cu(sk)
    need, room = _room(cu_q, cu_k, 2)
    assert need == 0 and room >= 65 * cu_q[-1] * 2 * 2 * 130 * 4   # of both maps' sums, maxima and sums of weights, in fp32


@pytest.mark.gpu
@pytest.mark.parametrize("late", [False, True])
@pytest.mark.parametrize("sq,sk", LONG)
def test_more_pieces_than_are_joined_at_a_time(sq, sk, late):
    """64 pieces are put together at a time.  The first map's largest score lies among the first keys and the second's among the last, or the other
    way round, so that what came before is scaled down by a later piece in one and kept in the other."""
    cu_q, cu_k = _cu(sq), _cu(sk)
    q, k, v, do, lam = _inputs(2, 128, torch.bfloat16, cu_q, cu_k, 51)
    for g in range(len(sq)):
        if sq[g] == 0:
            continue
        for m, s in enumerate((slice(0, 64), slice(64, 128))):
            at = cu_k[g] + 100 if (m == 0) != late else cu_k[g + 1] - 700
            k[:, at, s] = 1.3 * q[:, cu_q[g], s]   # a score of about 10, among others of 1.5 on average and 6.5 at most
    need, room = _room(cu_q, cu_k, 2)
    assert room > need
    _check(_run(q, k, v, do, lam, cu_q, cu_k, 0.125), q, k, v, do, lam, cu_q, cu_k, 0.125, near=False)
