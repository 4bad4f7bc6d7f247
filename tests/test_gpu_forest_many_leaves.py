"""Forests in 8 bits whose trees have more leaves together than one call takes."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def forest(n, trees, leaves_each, d_in, d_out, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d_in, generator=g).cuda()
    weight = torch.randn(trees * leaves_each, d_out, d_in, generator=g).cuda()
    bias = torch.randn(trees * leaves_each, d_out, generator=g).cuda()
    leaves = torch.randint(0, leaves_each, (n, trees), generator=g) + torch.arange(trees) * leaves_each
    return x, weight, bias, leaves.to(torch.int32).cuda(), torch.rand(n, trees, generator=g).cuda()


def answers(codes, x, leaves, gates):
    """In 64 bits, from the codes, a leaf's matrix gathered for every row; leaves outside are passed over."""
    c, s = ref.quantize(x)
    x64 = c.double() * s.double()[:, None]
    inside = (leaves >= 0) & (leaves < codes.weight.shape[0])
    at = torch.where(inside, leaves, 0).long()
    y, mag = 0.0, 0.0
    for j in range(leaves.shape[1]):
        w = codes.weight[at[:, j], :, :x.shape[1]].double() * codes.scales[at[:, j]].double()[:, :, None]
        b = codes.bias[at[:, j]].double()
        gate = torch.where(inside[:, j], gates[:, j].double(), 0.0)[:, None]
        y = y + gate * ((w * x64[:, None]).sum(2) + b)
        mag = mag + gate.abs() * ((w * x64[:, None]).abs().sum(2) + b.abs())
    return y, mag


@pytest.mark.parametrize("n", [1, 300])
@pytest.mark.parametrize("trees,leaves_each", [(65, 255), (100, 255), (3, 16_384), (130, 400), (2, 20_000)])
def test_trees_of_many_leaves(n, trees, leaves_each):
    """Sums of codes are exact: four roundings of a term, and one for each of at most `trees` + calls sums."""
    from paper_1706_08359_amd import routed_leaves as R
    x, weight, bias, leaves, gates = forest(n, trees, leaves_each, 11, 3, seed=trees)
    codes = R.Codes(weight, bias)
    want, mag = answers(codes, x, leaves, gates)
    got = codes.answer(x, leaves, gates)
    assert bool(((got.double() - want).abs() <= (2 * trees + 16) * U * mag).all())
    # leaves of any number in any slot, and none
    g = torch.Generator().manual_seed(n)
    leaves = torch.randint(-5, trees * leaves_each + 5, leaves.shape, generator=g).to(torch.int32).cuda()
    want, mag = answers(codes, x, leaves, gates)
    got = codes.answer(x, leaves, gates)
    assert bool(((got.double() - want).abs() <= (2 * trees + 16) * U * mag).all())


def test_rows_without_slots_are_refused():
    from paper_1706_08359_amd import routed_leaves as R
    x, weight, bias, leaves, gates = forest(4, 2, 3, 11, 3, seed=1)
    with pytest.raises(B.GbdtError):
        R.Codes(weight, bias).answer(x, leaves[:, :0], gates[:, :0])
