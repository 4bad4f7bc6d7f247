"""One row or one column out of something larger: the distance to the next one, which does not exist, is of no account."""
import pytest
import torch

from test_gpu_linear_leaves import make

pytestmark = pytest.mark.gpu


def far(t, distance):
    """The same row, of a matrix whose rows lie `distance` elements apart."""
    return t.as_strided(t.shape, (distance, 1))


def test_one_row_of_rows_that_lie_far_apart():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(1, [0, 1], 40, 24, "bf16", seed=1)
    y = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)
    grads = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    loss, lse = B.gbdt_softmax_loss(x, w[0], y)
    trained = B.gbdt_softmax_grad(x, w[0], y, lse)
    xf, dyf = far(x, 1 << 30), far(dy, (1 << 28) + 1)
    assert torch.equal(B.gbdt_leaf_product(xf, w, offs, row_idx=idx, bias=b), want)
    assert all(torch.equal(a, e) for a, e in zip(B.gbdt_leaf_product_grad(dyf, xf, w, offs, row_idx=idx), grads))
    got_loss, got_lse = B.gbdt_softmax_loss(xf, w[0], y)
    assert torch.equal(got_loss, loss) and torch.equal(got_lse, lse)
    assert all(torch.equal(a, e) for a, e in zip(B.gbdt_softmax_grad(xf, w[0], y, lse), trained))
    one = far(w[0][:1], 1 << 29)
    assert torch.equal(B.gbdt_softmax_loss(x, one)[1], B.gbdt_softmax_loss(x, w[0][:1])[1])


def test_one_column_of_statistics_into_larger_buffers():
    from paper_1706_08359_amd import binding as B
    x, _, w, _, _, _ = make(70, [70], 40, 24, "f32", seed=2)
    _, lse = B.gbdt_softmax_loss(x, w[0])
    want = B.gbdt_softmax_stats(x, w[0], None, lse, 7, 8)
    grads, hesses = torch.zeros(5, 100, device="cuda"), torch.zeros(5, 90, device="cuda")
    B.gbdt_softmax_stats(x, w[0], None, lse, 7, 8, grad_out=grads[2:3, :70], hess_out=hesses[4:5, 3:73])
    assert torch.equal(grads[2:3, :70], want[0]) and torch.equal(hesses[4:5, 3:73], want[1])
    grads[2], hesses[4] = 0.0, 0.0
    assert not bool(grads.any()) and not bool(hesses.any())
