"""Gradients of the weights over lists whose parts are longer than what a workgroup lists at once, and over more positions than
a launch has rows of workgroups for cuts of that length."""
import pytest
import torch

from oracle import linear_leaves as ref
from test_gpu_linear_leaves import close, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [5000, 4999])
@pytest.mark.parametrize("sizes", [[11_600, 0, 400], [100, 5900, 6000], [12_000]], ids=str)
def test_parts_longer_than_a_listing(sizes, d, dtype):
    """Matrices so large that only two cuts fit the scratch: 6,016 positions between them."""
    from paper_1706_08359_amd import binding as B
    need = B.gbdt_leaf_product_grad_workspace_bytes(12_000, d, d)
    assert need < 520 << 20
    x, dy, w, b, offs, idx = make(12_001, sizes, d, d, dtype, seed=len(sizes))
    idx[4090:4100:3], idx[6010:6020:4], idx[::997] = -1, 12_001, -5
    own = torch.empty(need, dtype=torch.uint8, device="cuda")
    B.gbdt_set_workspace(own)
    try:
        got = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight", "bias"))
        again = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight", "bias"))
        torch.cuda.synchronize()
    finally:
        B.gbdt_set_workspace(None)
    want, mags = ref.leaf_product_grad(dy, x, w, offs, idx, torch.zeros(12_001, 1, device="cuda").expand(12_001, d))
    for i in (1, 2):
        close(got[i], want[i], mags[i], max(sizes), i)
        assert torch.equal(got[i], again[i])


def test_more_positions_than_cuts_of_a_listing():
    """270 million positions of one input and one output.  Zeros and ones, a sum of which is below 2^24: every f32 sum is exact."""
    from paper_1706_08359_amd import binding as B
    n = 270_000_000
    g = torch.Generator(device="cuda").manual_seed(2)
    x = (torch.rand(n, 1, generator=g, device="cuda") < 0.05).float()
    dy = (torch.rand(n, 1, generator=g, device="cuda") < 0.05).float()
    edges = [0, 5, 150_000_001, 150_000_001, n]
    w = torch.zeros(4, 1, 1, device="cuda")
    _, dw, db = B.gbdt_leaf_product_grad(dy, x, w, torch.tensor(edges, device="cuda"), want=("weight", "bias"))
    for leaf in range(4):
        a, e = edges[leaf], edges[leaf + 1]
        assert int(dw[leaf, 0, 0]) == int((x[a:e] * dy[a:e]).double().sum())
        assert int(db[leaf, 0]) == int(dy[a:e].double().sum()) < 1 << 24


@pytest.mark.parametrize("d_out", [7_000_000, 7_000_001])
def test_outputs_sums_alone_of_wide_rows_fit_the_stated_scratch(d_out):
    """Sums of 7 million outputs: one matrix' sums would pass the scratch, so that the weights' gradient has one part; the outputs'
    alone have two.  The list names one row, of ones, 4,160 times (sums do not mind)."""
    from paper_1706_08359_amd import binding as B
    n = 4160
    dy = torch.ones(1, d_out, dtype=torch.bfloat16, device="cuda")
    idx, offs = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.tensor([0, n], device="cuda")
    got = torch.zeros(1, d_out, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.gbdt_leaf_product_grad_workspace_bytes(n, 8, d_out), dtype=torch.uint8, device="cuda")
    B.gbdt_set_workspace(ws)
    try:
        rc = B.load().gbdt_leaf_product_grad(dy.data_ptr(), d_out, None, 0, None, idx.data_ptr(), offs.data_ptr(), n, 1, 1, 8, d_out,
                                             1, None, 0, None, got.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    finally:
        B.gbdt_set_workspace(None)
    assert rc == 0 and bool((got == n).all())
