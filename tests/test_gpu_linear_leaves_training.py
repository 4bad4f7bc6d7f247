"""The calls together, as linear_leaves.Model uses them: a tree's row lists, its leaves' products, the loss and its gradients."""
import numpy as np
import pytest
import torch

from oracle import linear_leaves as ref

pytestmark = pytest.mark.gpu


def test_a_tree_routes_the_rows_its_products_are_grouped_by():
    from paper_1706_08359_amd import binding as B
    from paper_1706_08359_amd import linear_leaves as L
    x, bins, n_bins, labels, n_classes = L.synthetic(n_rows=3000, n_classes=40, seed=1)
    model = L.Model(x, bins, n_bins, labels, n_classes, dim=8)
    _, lse = model.loss()
    grad, hess = B.gbdt_softmax_stats(model.embed, model.classes, labels, lse, 0, 1)
    nodes, order, _ = B.gbdt_grow_tree(model.packed, 3000, 28, n_bins, grad[0], hess[0], 15, 1.0, 1e-3)
    leaves, offsets = L.leaf_lists(nodes, x.device)
    offs, rows = offsets.tolist(), order.cpu().numpy()
    assert len(leaves) == (len(nodes) + 1) // 2 and offs[0] == 0 and offs[-1] == 3000
    for i, leaf in enumerate(leaves):
        assert offs[i + 1] - offs[i] == nodes[leaf]["count"]
    routed, routed_offs = L.route(nodes, bins, leaves)
    assert routed_offs.tolist() == offs
    assert np.array_equal(routed.cpu().numpy(), rows)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 0.02)])
def test_one_step_is_the_formulas_step(dtype, tol):
    """The gradients of one step against the 64-bit definitions chained together.  f32: sums of at most 3,000 terms and a
    handful of roundings.  bf16: dh and the embeddings are rounded between the calls, 2^-8 each, beside the last rounding."""
    from paper_1706_08359_amd import binding as B
    from paper_1706_08359_amd import linear_leaves as L
    x, bins, n_bins, labels, n_classes = L.synthetic(n_rows=2000, n_classes=60, seed=2, dtype=dtype)
    labels[::9] = -1
    g = torch.Generator().manual_seed(3)
    order = torch.randperm(2000, generator=g).to(torch.int32).cuda()
    offs = torch.tensor([0, 700, 700, 1999, 2000], device="cuda")
    w = (0.3 * torch.randn(4, 16, 28, generator=g)).to(dtype).cuda()
    b = torch.randn(4, 16, generator=g).to(dtype).cuda()
    c = torch.randn(60, 16, generator=g).to(dtype).cuda()
    h = B.gbdt_leaf_product(x, w, offs, row_idx=order, bias=b)
    loss, lse = B.gbdt_softmax_loss(h, c, labels)
    dh, dc = B.gbdt_softmax_grad(h, c, labels, lse, scale=1 / 2000)
    dx, dw, db = B.gbdt_leaf_product_grad(dh, x, w, offs, row_idx=order)
    h64, _ = ref.leaf_product(x, w, b, offs, order, torch.zeros(2000, 16, device="cuda"))
    loss64, lse64 = ref.softmax_loss(h64, c, labels)
    (dh64, dc64), _ = ref.softmax_grad(h64, c, labels, lse64, None, 1 / 2000)
    (dx64, dw64, db64), _ = ref.leaf_product_grad(dh64, x, w, offs, order, torch.zeros(2000, 28, device="cuda"))
    for name, got, want in (("h", h, h64), ("loss", loss, loss64), ("dh", dh, dh64), ("dc", dc, dc64), ("dx", dx, dx64),
                            ("dw", dw, dw64), ("db", db, db64)):
        assert float((got.double() - want).norm()) <= tol * float(want.norm()), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_lowers_the_loss_and_predictions_agree(dtype):
    from paper_1706_08359_amd import linear_leaves as L
    x, bins, n_bins, labels, n_classes = L.synthetic(n_rows=6000, n_classes=100, seed=4, dtype=dtype)
    model = L.Model(x, bins, n_bins, labels, n_classes, dim=16)
    losses = [model.loss()[0]] + [model.add_tree(max_leaves=7, steps=12, rate=4.0) for _ in range(3)]
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    assert losses[-1] < losses[0] - 0.5
    assert torch.equal(model.embed_rows(x, bins), model.embed)
    p = model.probabilities(x[:1], bins[:1])
    assert p.shape == (n_classes, 1) and abs(float(p.sum()) - 1.0) < 1e-4
    few = model.embed_rows(x[:1], bins[:1])
    assert float((few.double() - model.embed[:1].double()).norm()) <= 0.02 * float(model.embed[:1].double().norm())
