"""Answers of several leaves whose outputs are of very different size, or that cancel: every output keeps its own digits.

u = 2^-24, half = half a step of the element type.  A result is a sum of d_in + 1 terms (dx: d_out) in f32, weighed and added up over
k slots in f32, rounded once: (d_in + k + 3) u of its own terms' magnitudes (codes, whose sums are exact: (k + 6) u) and half of
the result.  No term for the size of any other output, and none for answers that were rounded on the way."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B
from test_gpu_mixture import U, made

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def check(got, want, mag, roundings):
    half = torch.finfo(got.dtype).eps / 2
    bad = (got.double() - want).abs() > roundings * U * mag + half * want.abs()
    assert not bool(bad.any()) and not bool(torch.isnan(got).any()), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def check_all(x, dy, w, b, leaves, gates):
    """Answers and rows' gradients, and answers of codes in bf16."""
    (n_leaves, d_out, d_in), k = w.shape, leaves.shape[1]
    check(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), *ref.mixture(x, w, b, leaves, gates), d_in + k + 3)
    want, mag = ref.mixture_grad(dy, x, w, b, leaves, gates)
    dx, _, _, _ = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, want=("x",))
    check(dx, want[0], mag[0], d_out + k + 3)
    codes, scales = B.gbdt_rows_quantize(x)
    wc, ws = B.gbdt_rows_quantize(w.view(-1, d_in))
    wc, ws = wc.view(n_leaves, d_out, -1), ws.view(n_leaves, d_out)
    got = B.gbdt_mixture_product_codes(codes, scales, wc, ws, leaves, gates, bias=b.float(), dtype=x.dtype)
    check(got, *ref.mixture(codes.double() * scales.double()[:, None], wc.double() * ws.double()[:, :, None], b, leaves, gates), k + 6)


def ordinary(n, k, d_out, seed, d_in=64, n_leaves=4):
    """Weights of a row add up to at most 1."""
    x, dy, w, b, leaves, gates = made(n, k, n_leaves, d_in, d_out, "bf16", seed=seed)
    share = torch.rand(n, k, generator=torch.Generator().manual_seed(seed)).cuda() * 0.9 / k
    return x, dy, w, b, leaves, torch.where(torch.isnan(gates), gates, share)


@pytest.mark.parametrize("n,k", [(3, 3), (300, 2), (300, 9), (4000, 3)])
@pytest.mark.parametrize("size", [torch.finfo(BF16).min, 1e30, -1e12], ids=str)
def test_outputs_closed_by_a_bias(n, k, size):
    x, dy, w, b, leaves, gates = ordinary(n, k, 136, seed=n + k)
    b[:, 5] = size
    b[2, 130] = size
    check_all(x, dy, w, b, leaves, gates)


@pytest.mark.parametrize("n,k", [(3, 3), (300, 2), (300, 9), (20_000, 2)])
@pytest.mark.parametrize("size", [1e30, 1e12])
def test_a_large_output_and_a_large_input(n, k, size):
    """One row of every matrix, then one column (rows' gradients there are large, and x is nothing)."""
    x, dy, w, b, leaves, gates = ordinary(n, k, 136, seed=n - k)
    large = w.clone()
    large[:, 7] = (w[:, 7].float() * size).to(BF16)
    check_all(x, torch.where(torch.arange(136).cuda() == 7, 0.0, dy.float()).to(BF16), large, b, leaves, gates)
    large = w.clone()
    large[:, :, 9] = (w[:, :, 9].float() * size).to(BF16)
    x[:, 9] = 0.0
    want, mag = ref.mixture_grad(dy, x, large, b, leaves, gates)
    dx, _, _, _ = B.gbdt_mixture_product_grad(dy, x, large, leaves, gates, bias=b, want=("x",))
    check(dx, want[0], mag[0], 136 + k + 3)


@pytest.mark.parametrize("n", [3, 300, 9000])
def test_every_output_of_its_own_size(n):
    x, dy, w, b, leaves, gates = ordinary(n, 3, 128, seed=21)
    size = 2.0 ** torch.randint(-60, 60, (128,), generator=torch.Generator().manual_seed(1)).float().cuda()
    w, b = (w.float() * size[:, None]).to(BF16), (b.float() * size).to(BF16)
    check(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), *ref.mixture(x, w, b, leaves, gates), 64 + 3 + 3)


@pytest.mark.parametrize("n", [3, 300, 20_000])
@pytest.mark.parametrize("d_out", [66, 130, 258])
def test_a_large_first_output_and_the_last_ones(n, d_out):
    """The last columns of a tile that the outputs do not fill have nothing to do with the first output."""
    x, dy, w, b, leaves, gates = ordinary(n, 2, d_out, seed=d_out)
    w[:, 0] = (w[:, 0].float() * 2.0 ** 40).to(BF16)
    check(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), *ref.mixture(x, w, b, leaves, gates), 64 + 2 + 3)


@pytest.mark.parametrize("n", [3, 300])
def test_large_weights_beside_large_outputs(n):
    x, dy, w, b, leaves, gates = ordinary(n, 3, 72, seed=5)
    b[:, 3] = 1e30
    gates = gates * 2.0 ** 20
    check(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), *ref.mixture(x, w, b, leaves, gates), 64 + 3 + 3)


@pytest.mark.parametrize("n", [3, 300, 9000])
def test_answers_that_cancel(n):
    """Two leaves that differ by 2^-6 of their size, with weights 1 and -1: what is left has the digits of f32 sums."""
    x, dy, w, b, _, _ = made(n, 2, 2, 64, 128, "bf16", seed=8)
    w[1] = (w[0].float() * (1 + 2.0 ** -6)).to(BF16)
    b[1] = b[0]
    leaves = torch.tensor([[0, 1]], dtype=torch.int32).repeat(n, 1).cuda()
    gates = torch.tensor([[1.0, -1.0]]).repeat(n, 1).cuda()
    check_all(x, dy, w, b, leaves, gates)
