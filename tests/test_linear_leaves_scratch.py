"""Scratch of the linear-leaf and softmax calls does not grow with the number of rows or classes past its limits."""
import pytest
import torch

from paper_1706_08359_amd import binding as B

MIB = 1 << 20


@pytest.mark.parametrize("n,d_in,d_out", [(400_000, 2000, 256), (4_000_000, 2000, 256), (11_000_000, 2000, 256), (1 << 29, 700, 64),
                                          ((1 << 30) - 1, 1, 1), (1_000_000, 5000, 5000), (100_000, (1 << 24) - 1, 3)])
def test_sums_of_long_leaves_take_512_mib_at_most(n, d_in, d_out):
    assert 0 < B.gbdt_leaf_product_grad_workspace_bytes(n, d_in, d_out) <= 513 * MIB


def test_matrices_of_too_many_tiles_are_refused():
    """f32, 9 x 262,144 tiles of 64 x 64; refused before anything is enqueued, the gradient of the input too."""
    big = (1 << 24) - 1
    for dx in (None, 4096):
        assert B.load().gbdt_leaf_product_grad(4096, 513, 4096, big, 4096, None, 4096, 1, 1, 1, big, 513, 0, dx, big, 4096, None, None) == -2


@pytest.mark.parametrize("n", [4096, 100_000])
@pytest.mark.parametrize("v,dtype", [(4_000_000, torch.bfloat16), (10_000_000, torch.float32), (10_000_000, torch.bfloat16)])
def test_maxima_and_sums_of_millions_of_classes_take_few_rows_at_a_time(n, v, dtype):
    """The gradients' scratch, which the same number covers: G of 512 MiB or of 256 classes, f32 sums of dh and of a piece's dC, copies."""
    e, dim = (2 if dtype == torch.bfloat16 else 4), 8
    grad = max(512 * MIB, 256 * n * e) + 64 * MIB + 4 * n * dim * 4 + 16 * n + (v + n) * dim * e
    assert B.gbdt_softmax_workspace_bytes(n, v, dim, dtype) <= max(grad, 257 * MIB)
