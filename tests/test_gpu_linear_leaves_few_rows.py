"""A few rows of leaves with many outputs, on either side of where tiles take over."""
import pytest
import torch

from oracle import linear_leaves as ref
from test_gpu_linear_leaves import close, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[4], [5], [16], [17], [64], [2, 0, 1], [10, 6, 0, 16], [1] * 20, [0, 4, 0, 4, 0, 4, 0, 3]], ids=str)
@pytest.mark.parametrize("d_in,d_out", [(700, 1000), (137, 1025), (64, 3001), (3, 5000), (2000, 257)])
def test_many_outputs_of_few_rows(sizes, d_in, d_out, dtype):
    from paper_1706_08359_amd import binding as B
    rows = sum(sizes) + 2
    x, _, w, b, offs, idx = make(rows, sizes, d_in, d_out, dtype, seed=len(sizes))
    y0 = torch.full((rows, d_out), 5.0, dtype=x.dtype, device="cuda")
    y = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b, y_out=y0.clone())
    want, mag = ref.leaf_product(x, w, b, offs, idx, y0)
    close(y, want, mag, d_in, "y")
