"""Softmax gradients and leaf products at sizes that take the largest tiles over many steps, several pieces of classes with a split
sum, and lists of labels longer than a workgroup holds, against the definition in 64 bits."""
import pytest
import torch

from oracle import linear_leaves as ref
from test_gpu_linear_leaves import close
from test_gpu_softmax import check_grad, check_loss

pytestmark = pytest.mark.gpu


def make(n, v, dim, dtype, seed, few=None):
    """few: the labels of that share of the rows are among the first 256 classes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(n, dim, generator=g, device="cuda").to(dtype)
    c = (2.0 * dim ** -0.5 * torch.randn(v, dim, generator=g, device="cuda")).to(dtype)
    y = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    if few is not None:
        y = torch.where(torch.rand(n, generator=g, device="cuda") < few, y % min(v, 256), y)
    out = torch.rand(n, generator=g, device="cuda")
    y = torch.where(out < 0.05, torch.full_like(y, -1), torch.where(out < 0.1, torch.full_like(y, v), y))
    return h, c, y, torch.rand(n, generator=g, device="cuda") + 0.25


def exactness(h, c, y, w, scale, lse, got):
    """Root mean square errors, over those of the exact results rounded to the type."""
    want, _ = ref.softmax_grad(h, c, y, lse, w, scale)
    return [float((a.double() - e).norm()) / float((e.to(a.dtype).double() - e).norm()) for a, e in zip(got, want)]


@pytest.mark.parametrize("n,v,dim,few", [
    (1100, 33_000, 512, None),     # classes' gradient in tiles of 256 x 256, scores over 16 steps
    (4100, 33_000, 512, 0.5),      # the same with two thousand labels in its first tile
    (4090, 100_000, 505, None),    # two pieces, rows' gradient split eight ways in tiles of 256 x 256, copies of odd rows
    (8200, 40_000, 520, None),     # two pieces and splits, columns that end inside a tile
    (1400, 194_174, 40, None),     # two pieces and splits in tiles of 128 x 128
    (1600, 170_150, 40, None),     # the same, the last split of the shorter piece empty
    (20_000, 200, 4096, 0.9),      # more labels of a tile of 128 classes than a list holds
])
def test_large_bf16_gradients(n, v, dim, few):
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(n, v, dim, torch.bfloat16, v, few)
    _, lse = check_loss(B, h, c, y)
    got = check_grad(B, h, c, y, w, 1.0 / n, lse)
    again = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n)
    assert all(torch.equal(a, e) for a, e in zip(got, again))
    for want in ("h", "classes"):
        one = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n, want=(want,))
        assert torch.equal(one[0 if want == "h" else 1], got[0 if want == "h" else 1]) and one[1 if want == "h" else 0] is None
    for what, ratio in zip(("dh", "dc"), exactness(h, c, y, w, 1.0 / n, lse, got)):
        assert ratio <= 1.25, (what, ratio)


@pytest.mark.parametrize("n,v,dtype", [(300_000, 1700, torch.bfloat16), (160_000, 1700, torch.float32)])
def test_three_pieces_of_classes(n, v, dtype):
    """The scratch of both gradients is below half of what G takes, so the classes were taken in three pieces at least."""
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(n, v, 8, dtype, 3)
    assert B.gbdt_softmax_workspace_bytes(n, v, 8, dtype) < n * v * h.element_size() // 2
    _, lse = B.gbdt_softmax_loss(h, c, y)
    first = check_grad(B, h, c, y, w, 1.0 / n, lse)
    again = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n)
    assert all(torch.equal(a, e) for a, e in zip(first, again))
    only = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n, want=("h",))
    assert only[1] is None and torch.equal(only[0], first[0])
    only = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n, want=("classes",))
    assert only[0] is None and torch.equal(only[1], first[1])


@pytest.mark.parametrize("d_out", [100, 128, 200])
@pytest.mark.parametrize("d_in", [192, 520, 1032])
def test_long_leaves_over_many_steps(d_in, d_out):
    """Tiles of 256 rows, whose steps wait for some of the loads on their way (three stages; with more than 128 outputs four)."""
    from paper_1706_08359_amd import binding as B
    n = 66_100
    g = torch.Generator(device="cuda").manual_seed(d_in)
    x = torch.randn(n, d_in, generator=g, device="cuda").bfloat16()
    w, b = (torch.randn(5, d_out, k, generator=g, device="cuda").bfloat16() for k in (d_in, 1))
    idx = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    idx[::1001] = n
    offs = torch.tensor([0, 40_000, 40_000, 40_777, 66_000, 66_050], device="cuda")
    y0 = torch.full((n, d_out), 3.0, dtype=torch.bfloat16, device="cuda")
    y = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b[:, :, 0].contiguous(), y_out=y0.clone())
    want, mag = ref.leaf_product(x, w, b[:, :, 0], offs, idx, y0)
    close(y, want, mag, d_in, "y")
    assert torch.equal(y, B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b[:, :, 0].contiguous(), y_out=y0.clone()))
