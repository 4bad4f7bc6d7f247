"""More workgroups than one launch takes: it counts its threads in 32 bits, 16.7 million workgroups of 256."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

LEAVES = 8_500_000   # two column tiles of 64 each


def lists(n, seed):
    """n rows in leaves drawn from all, the first and the last among them."""
    g = torch.Generator().manual_seed(seed)
    leaf = torch.sort(torch.randint(0, LEAVES, (n,), generator=g))[0]
    leaf[:3], leaf[-2:] = 0, LEAVES - 1
    offs = torch.searchsorted(leaf, torch.arange(LEAVES + 1))
    return leaf.cuda(), torch.randperm(n, generator=g).to(torch.int32).cuda(), offs.cuda(), g


def test_product_of_millions_of_leaves():
    from paper_1706_08359_amd import binding as B
    n, d_out = 5000, 65
    leaf, idx, offs, g = lists(n, 1)
    x = torch.randn(n, 1, generator=g).cuda()
    w = torch.randn(LEAVES, d_out, 1, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    y = B.gbdt_leaf_product(x, w, offs, row_idx=idx, y_out=torch.full((n, d_out), 9.0, device="cuda"))
    rows = idx.long()
    want = w[leaf, :, 0].double() * x[rows].double()
    # one product, rounded once
    assert bool(((y[rows].double() - want).abs() <= 2.0 ** -24 * want.abs() + 1e-37).all())


def test_gradients_of_millions_of_leaves():
    from paper_1706_08359_amd import binding as B
    n, d_in = 5000, 65
    leaf, idx, offs, g = lists(n, 3)
    x, dy = torch.randn(n, d_in, generator=g).cuda(), torch.randn(n, 1, generator=g).cuda()
    w = torch.randn(LEAVES, 1, d_in, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    dx, dw, db = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    rows = idx.long()
    want = w[leaf, 0].double() * dy[rows].double()
    assert bool(((dx[rows].double() - want).abs() <= 2.0 ** -24 * want.abs() + 1e-37).all())
    used, at = torch.unique(leaf, return_inverse=True)
    each = dy[rows].double() * x[rows].double()
    sums = torch.zeros(len(used), d_in, dtype=torch.float64, device="cuda").index_add_(0, at, each)
    mags = torch.zeros_like(sums).index_add_(0, at, each.abs())
    # at most 20 rows a leaf: products and sums, each rounded
    assert int(torch.bincount(at).max()) <= 20
    assert bool(((dw[used, 0].double() - sums).abs() <= 23 * 2.0 ** -24 * mags).all())
    dys = torch.zeros(len(used), dtype=torch.float64, device="cuda").index_add_(0, at, dy[rows, 0].double())
    assert bool(((db[used, 0].double() - dys).abs() <= 23 * 2.0 ** -24 * 20 * dy.abs().max()).all())
    dw[used], db[used] = 0.0, 0.0
    assert not bool(dw.any()) and not bool(db.any())


def test_a_row_over_a_billion_classes():
    """Scores of 2^30 - 1 classes, f32: 2^24 tiles, eight of which are somebody's second."""
    from paper_1706_08359_amd import binding as B
    v = (1 << 30) - 1
    c = torch.zeros(v, 1, device="cuda")
    c[0], c[v // 2], c[v - 1] = 2.0, -3.0, 5.0
    h = torch.ones(1, 1, device="cuda")
    want = math.log(v - 3 + math.exp(2.0) + math.exp(-3.0) + math.exp(5.0))
    # 64 terms a part, then 65,536 parts a lane and 256 lanes: a relative error of 65,536 * 2^-24 at most, in the sum
    for y, s in ((v - 1, 5.0), (0, 2.0), (v // 2, -3.0), (12_345_678, 0.0)):
        loss, lse = B.gbdt_softmax_loss(h, c, torch.tensor([y], dtype=torch.int32, device="cuda"))
        assert abs(float(lse) - want) <= 0.005 and abs(float(loss) - (want - s)) <= 0.005
        assert abs(float(loss) - (float(lse) - s)) <= 4e-6
