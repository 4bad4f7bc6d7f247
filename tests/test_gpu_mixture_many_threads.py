"""Rows whose wavefronts, one for every few outputs, would be more threads than a launch counts in 32 bits: 56 GB of matrices."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu


def test_a_row_for_every_one_of_16384_leaves():
    torch.cuda.empty_cache()
    n, d_in, d_out = 16_384, 104, 8192
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(n, d_out, d_in, device="cuda")
    for a in range(0, n, 1024):
        w[a:a + 1024].normal_(generator=g)
    x = torch.randn(n, d_in, generator=g, device="cuda")
    leaves = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
    gates = torch.rand(n, 1, generator=g, device="cuda")
    y = B.gbdt_mixture_product(x, w, leaves, gates)
    for d in (0, 1, n // 2, n - 2, n - 1):
        want, mag = ref.mixture(x[d:d + 1], w[leaves[d].long()], None, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), gates[d:d + 1])
        assert bool(((y[d:d + 1].double() - want).abs() <= (d_in + 5) * 2.0 ** -24 * mag).all()), d
    assert bool((y != 0).any(1).all())
    del w, y
    torch.cuda.empty_cache()
