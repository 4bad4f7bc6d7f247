"""Products of codes whose sum times one scale leaves the 32-bit numbers while the result does not."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,k", [(2, 1), (3, 3), (300, 1), (300, 3), (70_000, 1)])
@pytest.mark.parametrize("rows,matrices", [(2e36, 1e-33), (1e-33, 2e36), (1e-37, 1e35), (1e35, 1e-37)])
def test_scales_far_apart(dtype, n, k, rows, matrices):
    """Sums of 200 codes are up to 3.2 million.  Results: the conversion, two products, the bias, weight and sum over k: (k + 6) u of the
    magnitudes, and half a step."""
    g = torch.Generator().manual_seed(n + k)
    codes = torch.zeros(n, 208, dtype=torch.int8)
    codes[:, :200] = torch.randint(-127, 128, (n, 200), generator=g)
    w = torch.zeros(5, 72, 208, dtype=torch.int8)
    w[:, :, :200] = torch.randint(-127, 128, (5, 72, 200), generator=g)
    scales = (torch.rand(n, generator=g) + 0.2) * rows
    ws = (torch.rand(5, 72, generator=g) + 0.2) * matrices
    scales[1], ws[2, 3] = float("nan"), float("nan")
    b = torch.randn(5, 72, generator=g)
    leaves = torch.randint(0, 5, (n, k), generator=g, dtype=torch.int32)
    gates = torch.rand(n, k, generator=g)
    codes, w, scales, ws, b, leaves, gates = (t.cuda() for t in (codes, w, scales, ws, b, leaves, gates))
    want, mag = ref.mixture(codes.double() * scales.double()[:, None], w.double() * ws.double()[:, :, None], b, leaves, gates)
    got = B.gbdt_mixture_product_codes(codes, scales, w, ws, leaves, gates, bias=b, dtype=dtype)
    half = torch.finfo(dtype).eps / 2

    def check(got, want, mag):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = (got.double() - want).abs() <= (k + 6) * U * mag + half * want.abs()
        assert bool((ok | torch.isnan(want)).all())
    check(got, want, mag)
    if k == 1:
        order = torch.sort(leaves[:, 0], stable=True)[1].to(torch.int32)
        offsets = torch.zeros(6, dtype=torch.int64).cuda()
        offsets[1:] = torch.cumsum(torch.bincount(leaves[:, 0].long(), minlength=5), 0)
        got = B.gbdt_leaf_product_codes(codes, scales, w, ws, offsets, row_idx=order, bias=b, dtype=dtype)
        check(got, *ref.mixture(codes.double() * scales.double()[:, None], w.double() * ws.double()[:, :, None], b, leaves,
                                torch.ones_like(gates)))
