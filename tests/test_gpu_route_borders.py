"""Borders between groups that 32 bits cannot draw: pairs of choice values that nearly cancel, leaves closed by a lowest value as their
bias, scores that are saturated.  Chosen leaves equal those of the definition in 64 bits."""
import math

import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu


def nearly_tied(n, n_groups, group_size, score, size, seed):
    """Logits, and biases that give each group two open leaves of opposite sign, about size, whose values add up to nearly the same
    in all groups; the group's other leaves are closed by their logits."""
    g = torch.Generator().manual_seed(seed)
    row = torch.randn(1, n_groups * group_size, generator=g)
    row.view(n_groups, group_size)[:, 2:] = -math.inf
    s = ref.scores(row, score)[0].view(n_groups, group_size)
    bias = torch.zeros(n_groups, group_size)
    up = torch.rand(n_groups, generator=g) < 0.5
    first = (size * (1 + 0.25 * torch.rand(n_groups, generator=g))) * torch.where(up, 1.0, -1.0)
    bias[:, 0] = first
    bias[:, 1] = (0.03 - s[:, 0] - s[:, 1] - first.double()).float()
    l = row.repeat(n, 1)
    l[1:] += torch.randn(n - 1, l.shape[1], generator=g) * size * 1e-7
    return l, bias.view(-1)


def group_values(l, bias, score, n_groups):
    c = ref.scores(l, score)[0] + bias.double()
    c = torch.where(l.double() == -math.inf, -math.inf, c).view(l.shape[0], n_groups, -1)
    return torch.sort(c, 2, descending=True)[0][:, :, :2].sum(2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [17.0, 110.0, 1000.0])
@pytest.mark.parametrize("n_groups,group_size,kept", [(32, 2, 6), (8, 8, 3), (16, 16, 5), (4, 16, 2), (12, 32, 4), (64, 16, 16)])
def test_two_best_values_that_cancel(score, size, n_groups, group_size, kept):
    l, bias = nearly_tied(400, n_groups, group_size, score, size, seed=n_groups)
    worth = torch.sort(group_values(l, bias, score, n_groups), 1, descending=True)[0]
    gap = worth[:, kept - 1] - worth[:, kept]
    told = gap > 1e-11 * size   # what 64 bits tell apart
    assert int(told.sum()) > 390 and float(gap.median()) < 1e-6 * size
    how = dict(score=score, n_groups=n_groups, groups_kept=kept, group_best=2)
    leaves, _ = B.gbdt_route(l.cuda(), 2 * kept, choice_bias=bias.cuda(), **how)
    want, _ = ref.route(l, 2 * kept, choice_bias=bias, **how)
    # (both leaves of a kept group are taken, so groups alone decide; the order of leaves of nearly equal values is another matter)
    leaves, want = torch.sort(leaves.cpu(), 1)[0], torch.sort(want, 1)[0]
    wrong = (leaves != want).any(1) & told
    assert not bool(wrong.any()), int(wrong.sum())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, -2e38], ids=str)
@pytest.mark.parametrize("n_groups,group_size", [(8, 8), (8, 3), (8, 16), (16, 32), (6, 2)])
def test_groups_closed_by_the_lowest_value(score, low, n_groups, group_size):
    """Two groups are open, one has a single open leaf, the others are closed by a bias whose double leaves the 32-bit numbers: they
    come after all others, the lowest first, and are taken where more groups are kept than are open."""
    g = torch.Generator().manual_seed(group_size)
    l = torch.randn(50, n_groups * group_size, generator=g)
    bias = torch.full((n_groups, group_size), low)
    bias[1], bias[n_groups - 1] = 0.1, 0.0
    bias[3, 1] = 0.2
    bias = bias.view(-1)
    for kept in (2, 3, 4, n_groups):
        how = dict(score=score, n_groups=n_groups, groups_kept=kept, group_best=2)
        k = min(32, kept * group_size)
        leaves, gates = B.gbdt_route(l.cuda(), k, choice_bias=bias.cuda(), **how)
        want, want_gates = ref.route(l, k, choice_bias=bias, **how)
        assert torch.equal(leaves.cpu(), want), kept
        assert bool((leaves >= 0).all())
        assert bool(((gates.cpu().double() - want_gates).abs() <= 1e-4 * want_gates.abs() + 1e-37).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_groups,group_size,kept", [(4, 4, 2), (8, 8, 3), (4, 64, 2), (3, 43, 1), (16, 32, 5)])
def test_without_a_bias_the_order_is_that_of_the_logits(score, dtype, n_groups, group_size, kept):
    """Sigmoids of logits from 37 on are all 1 in 64 bits, softmaxes of those 745 below the largest all 0: in the groups that their two
    best scores keep, leaves are taken by their logits all the same."""
    g = torch.Generator().manual_seed(group_size)
    n = n_groups * group_size
    l = (torch.randperm(n, generator=g)[None] * torch.ones(40, 1) * 0.5 + 38.0)
    l[10:20] = torch.randperm(n, generator=g) * -900.0
    l[20:30] = torch.randn(10, n, generator=g) * 30 + 40
    l[30:] = torch.randn(10, n, generator=g) * 600
    l = torch.where((l > 28) & (l < 38.5), l + 11, l).to(dtype)   # (between, sigmoids differ from 1 by a last place or two)
    how = dict(score=score, n_groups=n_groups, groups_kept=kept, group_best=2)
    k = min(32, kept * group_size)
    leaves, gates = B.gbdt_route(l.cuda(), k, **how)
    leaves = leaves.cpu().long()
    took = l.double().gather(1, leaves)
    assert bool((took[:, 1:] <= took[:, :-1]).all())
    want, _ = ref.route(l, k, **how)
    assert torch.equal(leaves, want.long())


@pytest.mark.parametrize("n_groups,group_size", [(8, 8), (6, 2), (8, 32)])
def test_values_of_opposite_sign_whose_sizes_leave_the_numbers(n_groups, group_size):
    """3e38 and -3e38 add up to what their scores leave, and their sizes to more than f32 holds: 64 bits alone can tell the groups apart."""
    g = torch.Generator().manual_seed(n_groups)
    l = torch.randn(60, n_groups * group_size, generator=g)
    l.view(60, n_groups, group_size)[:, :, 2:] = -math.inf
    bias = torch.zeros(n_groups, group_size)
    bias[:, 0] = 3e38 * (1 - 2.0 ** -10 * torch.rand(n_groups, generator=g))
    bias[:, 1] = -bias[:, 0] * (1 + 2.0 ** -20 * torch.randint(-3, 4, (n_groups,), generator=g))
    bias[n_groups - 1, :2] = torch.finfo(torch.float32).min
    bias = bias.view(-1)
    for kept in (1, 2, n_groups - 1, n_groups):
        how = dict(score="sigmoid", n_groups=n_groups, groups_kept=kept, group_best=2)
        leaves, _ = B.gbdt_route(l.cuda(), 2 * kept, choice_bias=bias.cuda(), **how)
        want, _ = ref.route(l, 2 * kept, choice_bias=bias, **how)
        assert torch.equal(leaves.cpu(), want), kept
