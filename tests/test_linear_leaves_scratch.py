"""Scratch of the linear-leaf and softmax calls does not grow with the number of rows or classes past its limits."""
import pytest

from paper_1706_08359_amd import binding as B

MIB = 1 << 20


@pytest.mark.parametrize("n,d_in,d_out", [(400_000, 2000, 256), (4_000_000, 2000, 256), (11_000_000, 2000, 256), (1 << 29, 700, 64),
                                          ((1 << 30) - 1, 1, 1), (1_000_000, 5000, 5000), (100_000, (1 << 24) - 1, 3)])
def test_sums_of_long_leaves_take_512_mib_at_most(n, d_in, d_out):
    assert 0 < B.gbdt_leaf_product_grad_workspace_bytes(n, d_in, d_out) <= 513 * MIB
