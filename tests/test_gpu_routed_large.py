"""Matrices of more than 4 GiB: rows whose places pass 32 bits, checked where they lie first and last."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def ends(n, some=700):
    return torch.cat([torch.arange(some), torch.arange(n // 2, n // 2 + 50), torch.arange(n - some, n)]).cuda()


def test_rows_of_4_gib():
    n, d_in, d_out, k, n_leaves = 1_200_000, 2000, 8, 2, 5
    x = torch.zeros(n, d_in, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for a in range(0, n, 100_000):
        x[a:a + 100_000] = torch.randn(100_000, d_in, generator=g, device="cuda")
    w = (torch.randn(n_leaves, d_out, d_in, generator=g, device="cuda") * d_in ** -0.5).to(torch.bfloat16)
    leaves = torch.randint(0, n_leaves, (n, k), generator=g, device="cuda", dtype=torch.int32)
    gates = torch.rand(n, k, generator=g, device="cuda")
    at = ends(n)
    y = B.gbdt_mixture_product(x, w, leaves, gates)
    want, mag = ref.mixture(x[at], w, None, leaves[at], gates[at])
    tol = (d_in + k + 3) * U * mag + 2.0 ** -8 * want.abs() + 2.0 ** -11 * mag + 2.0 ** -39 * mag.amax(1, keepdim=True)
    assert bool(((y[at].double() - want).abs() <= tol).all())
    dy = torch.randn(n, d_out, generator=g, device="cuda").to(torch.bfloat16)
    dx, _, _, dg = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("x", "gates"))
    (dx64, _, _, dg64), (dx_mag, _, _, dg_mag) = ref.mixture_grad(dy[at], x[at], w, None, leaves[at], gates[at])
    tol = (d_out + k + 3) * U * dx_mag + 2.0 ** -8 * dx64.abs() + 2.0 ** -11 * dx_mag + 2.0 ** -39 * dx_mag.amax(1, keepdim=True)
    assert bool(((dx[at].double() - dx64).abs() <= tol).all())
    assert bool(((dg[at].double() - dg64).abs() <= (d_in + 2 * d_out + 4) * U * dg_mag).all())


def test_codes_of_4_gib():
    n, d_in, d_out = 2_200_000, 2000, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    codes = torch.randint(-127, 128, (n, d_in), generator=g, device="cuda", dtype=torch.int8)
    scales = torch.rand(n, generator=g, device="cuda") + 0.1
    w = torch.randint(-127, 128, (3, d_out, d_in), generator=g, device="cuda", dtype=torch.int8)
    ws = torch.rand(3, d_out, generator=g, device="cuda")
    offs = torch.tensor([0, 700_000, 1_500_000, n], device="cuda")
    y = B.gbdt_leaf_product_codes(codes, scales, w, ws, offs)
    at = ends(n)
    leaf = torch.bucketize(at, offs[1:-1], right=True).to(torch.int32)[:, None]
    want, mag = ref.mixture(codes[at].double() * scales[at].double()[:, None], w.double() * ws.double()[:, :, None], None, leaf,
                            torch.ones_like(leaf, dtype=torch.float32))
    assert bool(((y[at].double() - want).abs() <= 5 * U * mag).all())


def test_logits_of_4_gib():
    n = 4_300_000
    g = torch.Generator(device="cuda").manual_seed(3)
    l = torch.empty(n, 255, device="cuda")
    for a in range(0, n, 430_000):
        l[a:a + 430_000] = torch.randn(430_000, 255, generator=g, device="cuda")
    leaves, gates = B.gbdt_route(l, 3)
    at = ends(n)
    want, want_gates = ref.route(l[at], 3)
    assert torch.equal(leaves[at], want)
    assert bool(((gates[at].double() - want_gates).abs() <= 300 * U * want_gates).all())
    dg = torch.ones(n, 3, device="cuda")
    dg[:, 0] = 2.0
    d = B.gbdt_route_grad(l, leaves, dg, renormalise=False)
    want, mag = ref.route_grad(l[at], leaves[at], dg[at], renormalise=False)
    assert bool(((d[at].double() - want).abs() <= 320 * U * mag + U * want.abs()).all())
