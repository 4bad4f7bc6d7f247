"""Routing on the GPU against the definition in 64 bits: chosen leaves equal, weights and gradients within bounds of their roundings.

u = 2^-24.  A score is an exponential (the argument's rounding, |l - top| u, and 2 u of the function) over a sum of at most n_leaves
of them; a weight is at most two such quotients and the scale: (n_leaves + 16 + 2 span) u of its size, span the spread of the finite
logits.  The gradient adds a sum over k and four products: (n_leaves + k + 24 + 4 span) u of its terms' magnitudes, and its rounding to
the logits' type."""
import math

import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def made(n, n_leaves, dtype, seed, masked=0.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(n, n_leaves, generator=g) * 1.5
    if masked:
        l[torch.rand(n, n_leaves, generator=g) < masked] = -math.inf
        l[torch.rand(n, n_leaves, generator=g) < masked / 4] = math.nan
    buf = torch.full((n, n_leaves + pad), 7.0, dtype=DTYPES[dtype]).cuda()
    buf[:, :n_leaves] = l.to(DTYPES[dtype]).cuda()
    return buf[:, :n_leaves], g


def span(l):
    f = l.double()
    f = f[torch.isfinite(f)]
    return float(f.max() - f.min()) if f.numel() else 0.0


def check(l, k, dgates, bias=None, score="softmax", renormalise=True, scale=1.0, **groups):
    how = dict(score=score, renormalise=renormalise, scale=scale)
    leaves, gates = B.gbdt_route(l, k, choice_bias=bias, **how, **groups)
    want, want_gates = ref.route(l, k, choice_bias=bias, **how, **groups)
    assert torch.equal(leaves, want)
    n = l.shape[1]
    tol = (n + 16 + 2 * span(l)) * U
    assert bool(((gates.double() - want_gates).abs() <= tol * want_gates.abs() + 1e-37).all())
    d = B.gbdt_route_grad(l, leaves, dgates, **how)
    assert d.dtype == l.dtype and d.shape == l.shape
    want_d, mag = ref.route_grad(l, leaves, dgates, **how)
    half = torch.finfo(l.dtype).eps / 2
    tol = (n + k + 24 + 4 * span(l)) * U
    assert bool(((d.double() - want_d).abs() <= tol * mag + half * want_d.abs() + 1e-37).all())
    return leaves, gates, d


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,n_leaves,k", [(1, 1, 1), (1, 255, 2), (7, 2, 2), (33, 8, 3), (65, 31, 31), (100, 32, 4), (31, 33, 5),
                                          (50, 64, 8), (29, 65, 1), (30, 128, 16), (19, 137, 3), (257, 256, 8), (9, 257, 4),
                                          (6, 512, 32), (5, 513, 6), (3, 1023, 7), (4, 1024, 32)])
def test_sizes(score, renormalise, dtype, n, n_leaves, k):
    l, g = made(n, n_leaves, dtype, seed=n * 1000 + n_leaves, pad=n_leaves % 3)
    dg = torch.randn(n, k, generator=g).cuda()
    check(l, k, dg, score=score, renormalise=renormalise, scale=2.5)
    bias = (torch.randn(n_leaves, generator=g) * 0.1).cuda()
    check(l, k, dg, bias=bias, score=score, renormalise=renormalise)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("n,n_leaves,groups,kept,k", [(40, 256, 8, 4, 8), (17, 64, 64, 5, 5), (23, 24, 3, 1, 8), (11, 130, 2, 1, 9),
                                                      (9, 1024, 32, 3, 4), (13, 12, 4, 4, 12), (50, 6, 3, 2, 3), (8, 640, 64, 9, 32)])
def test_groups(score, best, with_bias, n, n_leaves, groups, kept, k):
    l, g = made(n, n_leaves, "f32", seed=n_leaves + kept, masked=0.1)
    dg = torch.randn(n, k, generator=g).cuda()
    bias = (torch.randn(n_leaves, generator=g) * 0.2).cuda() if with_bias else None
    check(l, k, dg, bias=bias, score=score, n_groups=groups, groups_kept=kept, group_best=best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("n_leaves,k", [(8, 6), (40, 8), (255, 4)])
def test_masked_leaves(score, renormalise, n_leaves, k):
    """Most leaves closed, whole rows among them: slots that nothing is left for, and NaN in their gradients."""
    l, g = made(90, n_leaves, "f32", seed=5, masked=0.9)
    l[3] = -math.inf
    l[4] = math.nan
    dg = torch.randn(90, k, generator=g).cuda()
    leaves, gates = B.gbdt_route(l, k)
    assert int((leaves < 0).sum()) > 0 and bool((leaves[3:5] == -1).all()) and bool((gates[3:5] == 0).all())
    dg = torch.where(leaves < 0, math.nan, dg)
    _, _, d = check(l, k, dg, score=score, renormalise=renormalise)
    assert bool((d[3:5] == 0).all()) and bool(torch.isfinite(d).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_values_go_to_the_lowest_leaf(score):
    l = torch.zeros(70, 255).cuda()
    l[:, 9::50] = 1.0
    leaves, _ = B.gbdt_route(l, 8, score=score)
    assert leaves.tolist() == [[9, 59, 109, 159, 209, 0, 1, 2]] * 70
    leaves, _ = B.gbdt_route(l, 8, score=score, choice_bias=torch.zeros(255).cuda())
    assert leaves.tolist() == [[9, 59, 109, 159, 209, 0, 1, 2]] * 70
    l = torch.randint(0, 3, (200, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    check(l, 12, torch.ones(200, 12).cuda(), score=score, bias=torch.zeros(64).cuda())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [dict(), dict(n_groups=8, groups_kept=3, group_best=2)])
def test_values_closer_than_32_bits_hold(score, groups):
    """A bias that makes all choice values of a row nearly equal: their order is that of 64 bits."""
    g = torch.Generator().manual_seed(11)
    row = torch.randn(1, 64, generator=g)
    s, _ = ref.scores(row, score)
    bias = (0.75 - s[0]).float().cuda()
    l = row.repeat(90, 1).cuda()
    l[1::2] += torch.randn(45, 64, generator=g).cuda() * 1e-7
    c = torch.sort(ref.scores(l, score)[0] + bias.double(), dim=1)[0]
    assert float((c[:, 1:] - c[:, :-1]).max()) < 1e-6
    check(l, 8, torch.randn(90, 8, generator=g).cuda(), bias=bias, score=score, **groups)


def test_infinite_logits_and_biases():
    inf = math.inf
    l = torch.tensor([[inf, 1.0, inf, 2.0, -inf, 0.0], [-3e38, 3e38, 0.0, 3e38, -inf, 1.0], [-200.0, -201.0, -200.5, -230.0, -900.0, -250.0]]).cuda()
    for score in ("softmax", "sigmoid"):
        leaves, gates = B.gbdt_route(l, 2, score=score)
        assert leaves.tolist() == [[0, 2], [1, 3], [0, 2]] and gates[:2].tolist() == [[0.5, 0.5]] * 2
        share = torch.softmax(torch.tensor([-200.0, -200.5]).double(), 0)
        assert torch.allclose(gates[2].cpu().double(), share, rtol=1e-6)
    bias = torch.tensor([0.0, inf, -inf, math.nan, 0.0, inf]).cuda()
    leaves, _ = B.gbdt_route(l[:1], 4, choice_bias=bias, score="sigmoid")
    assert leaves.tolist() == [[1, 5, 0, -1]]


def test_leaves_named_twice_or_outside_in_the_gradient():
    l, g = made(20, 40, "f32", seed=2)
    leaves = torch.randint(-3, 44, (20, 6), generator=g, dtype=torch.int32).cuda()
    leaves[:, 1] = leaves[:, 0]
    leaves[0] = 99
    dg = torch.randn(20, 6, generator=g).cuda()
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            got = B.gbdt_route_grad(l, leaves, dg, score=score, renormalise=renormalise)
            want, mag = ref.route_grad(l, leaves, dg, score=score, renormalise=renormalise)
            assert bool(((got.double() - want).abs() <= (40 + 6 + 24 + 4 * span(l)) * U * mag + U * want.abs()).all())


def test_gradient_against_differences():
    """Central differences of the GPU's own weights, choice unchanged: h = 2^-6 leaves h^2 / 6 of a third derivative (below 1 for
    these scores) and the weights' roundings over h."""
    l, g = made(6, 12, "f32", seed=4)
    dg = torch.randn(6, 12, generator=g).cuda()
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            how = dict(score=score, renormalise=renormalise)

            def weights(v):
                """By leaf, all twelve chosen, so that no order matters."""
                leaves, gates = B.gbdt_route(v, 12, **how)
                return torch.zeros(6, 12).cuda().scatter_(1, leaves.long(), gates)
            leaves = torch.arange(12, dtype=torch.int32).repeat(6, 1).cuda()
            got = B.gbdt_route_grad(l, leaves, dg, **how)
            h = 2.0 ** -6
            for e in range(12):
                step = torch.zeros(6, 12).cuda()
                step[:, e] = h
                diff = ((weights(l + step) - weights(l - step)) * dg).sum(1) / (2 * h)
                assert float((diff - got[:, e]).abs().max()) <= h * h / 6 * float(dg.abs().sum(1).max()) + 64 * U / h * float(dg.abs().sum(1).max())


def test_rows_past_the_batch_are_left_alone_and_many_rows():
    l, g = made(70_001, 33, "bf16", seed=8, pad=1)
    leaves = torch.full((70_005, 4), 77, dtype=torch.int32).cuda()
    gates = torch.full((70_005, 4), 77.0).cuda()
    B.gbdt_route(l, 4, leaves_out=leaves[:70_001], gates_out=gates[:70_001])
    assert bool((leaves[70_001:] == 77).all()) and bool((gates[70_001:] == 77).all())
    want, _ = ref.route(l, 4)
    assert torch.equal(leaves[:70_001], want)
    out = torch.full((70_001, 40), 5.0, dtype=torch.bfloat16).cuda()
    B.gbdt_route_grad(l, leaves[:70_001], torch.ones(70_001, 4).cuda(), renormalise=False, dlogits_out=out[:, 3:36])
    assert bool((out[:, :3] == 5).all()) and bool((out[:, 36:] == 5).all())
    empty = torch.zeros(0, 33, dtype=torch.bfloat16).cuda()
    assert B.gbdt_route(empty, 4)[0].shape == (0, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_types_lowest_value_as_a_mask(dtype):
    """Leaves closed by the lowest finite value have no weight, and a row of nothing else is shared evenly."""
    l, g = made(40, 70, dtype, seed=3)
    low = torch.finfo(DTYPES[dtype]).min
    l[:, 5:60] = low
    l[7] = low
    for score in ("softmax", "sigmoid"):
        leaves, gates = B.gbdt_route(l, 20, score=score)
        want, want_gates = ref.route(l, 20, score=score)
        assert torch.equal(leaves, want)
        assert float((gates.double() - want_gates).abs().max()) <= 1e-6 and bool(torch.isfinite(gates).all())
        assert bool((gates[7] == gates[7, 0]).all()) and abs(float(gates[7].sum()) - 1.0) < 1e-5
        d = B.gbdt_route_grad(l, leaves, torch.randn(40, 20, generator=g).cuda(), score=score)
        assert bool(torch.isfinite(d).all())
