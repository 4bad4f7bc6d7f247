"""Gradients of the biases where a leaf's weighted rows cancel: sums of f32 products, whatever the element type.

u = 2^-24.  A term is one product in f32, a leaf has up to n k of them: (n k + 2) u of the magnitudes, and half a step of the result."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B
from test_gpu_mixture import U, made

pytestmark = pytest.mark.gpu


def check(db, dy, x, w, leaves, gates):
    want, mag = ref.mixture_grad(dy, x, w, None, leaves, gates)
    half = torch.finfo(db.dtype).eps / 2
    bad = (db.double() - want[2]).abs() > (leaves.numel() + 2) * U * mag[2] + half * want[2].abs()
    assert not bool(bad.any()) and not bool(torch.isnan(db).any()), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 8, 1, 0), (6, 2, 3, 8, 33, 0), (300, 3, 4, 16, 130, 3), (700, 9, 40, 16, 7, 1), (20_000, 2, 3, 64, 100, 0),
                                  (400, 2, 5000, 8, 8, 0), (60_000, 1, 2, 8, 20, 0), (3000, 4, 1, 128, 1000, 0)], ids=str)
@pytest.mark.parametrize("want", [("bias",), ("weight", "bias"), ("x", "weight", "bias", "gates")], ids=str)
def test_rows_that_cancel(dtype, size, want):
    """The second half of the rows is the first with the gates' signs turned, but for 2^-7 of them."""
    n, k, n_leaves, d_in, d_out, pad = size
    x, dy, w, b, leaves, gates = made(n, k, n_leaves, d_in, d_out, dtype, seed=n + d_out, pad=pad)
    h = n // 2
    dy[n - h:], leaves[n - h:], gates[n - h:] = dy[:h], leaves[:h], gates[:h] * (2.0 ** -7 - 1)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, want=want)
    check(got[2], dy, x, w, leaves, gates)
    again = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, want=want)
    assert torch.equal(got[2], again[2])


def test_rows_of_no_leaf_are_not_read():
    x, dy, w, b, leaves, gates = made(500, 3, 6, 16, 40, "bf16", seed=4)
    leaves[7] = -1
    dy[7] = float("nan")
    db = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("bias",))[2]
    dy[7] = 0.0
    check(db, dy, x, w, leaves, gates)
