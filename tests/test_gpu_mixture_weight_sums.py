"""Gradients of the matrices where a leaf's weighted rows cancel.

u = 2^-24.  f32: a term is two products, a leaf has up to n k of them: (n k + 3) u of the magnitudes.  bf16: gates * dy (u) is the sum of two
values.  Of a v between 2^E and 2^(E + 1) the first, of 8 bits, is off by 2^(E - 8) at most; the second, of what is left, by half a step of a number
below 2^(E - 8), 2^(E - 17): 2^-17 of every term, and sums of twice as many exact products: 2^-17 + (2 n k + 3) u.  And half a step of the
result."""
import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B
from test_gpu_mixture import U, made

pytestmark = pytest.mark.gpu


def check(dw, dy, x, w, leaves, gates, but=None):
    want, mag = ref.mixture_grad(dy, x, w, None, leaves, gates)
    if but is not None:
        want[1][but] = 0.0
    half, short = torch.finfo(dw.dtype).eps / 2, dw.dtype != torch.float32
    tol = 2.0 ** -17 + (2 * leaves.numel() + 3) * U if short else (leaves.numel() + 3) * U
    bad = (dw.double() - want[1]).abs() > tol * mag[1] + half * want[1].abs()
    assert not bool(bad.any()) and not bool(torch.isnan(dw).any()), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 8, 1, 0), (2, 1, 1, 9, 3, 0), (6, 2, 3, 8, 33, 0), (300, 3, 4, 137, 130, 3), (700, 2, 40, 16, 7, 1),
                                  (900, 1, 3, 264, 300, 0), (2100, 1, 1, 24, 64, 0), (300, 2, 5000, 8, 8, 0), (450, 2, 2, 40, 200, 8)], ids=str)
def test_rows_that_cancel(dtype, size):
    """The second half of the rows is the first with the gates' signs turned, but for 2^-7 of them."""
    n, k, n_leaves, d_in, d_out, pad = size
    x, dy, w, b, leaves, gates = made(n, k, n_leaves, d_in, d_out, dtype, seed=n + d_out, pad=pad)
    h = n // 2
    x[n - h:], dy[n - h:], leaves[n - h:], gates[n - h:] = x[:h], dy[:h], leaves[:h], gates[:h] * (2.0 ** -7 - 1)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("weight",))
    check(got[1], dy, x, w, leaves, gates)
    again = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b)
    assert torch.equal(got[1], again[1])


@pytest.mark.parametrize("d_in", [64, 63])
def test_weights_of_every_size(d_in):
    """Gates of 2^-40 to 2^40, and one that makes gates * dy infinite in its row of dy alone."""
    x, dy, w, b, leaves, gates = made(500, 2, 4, d_in, 72, "bf16", seed=3, outside=0.0)
    gates = gates * 2.0 ** torch.randint(-40, 41, gates.shape, generator=torch.Generator().manual_seed(1)).float().cuda()
    check(B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("weight",))[1], dy, x, w, leaves, gates)
    dy[5, 3], gates[5, 0], leaves[5, 0] = 2.0 ** 100, 2.0 ** 100, 1
    dw = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("weight",))[1]
    assert bool(torch.isinf(dw[1, 3]).all())
    # (the row's other leaf has the same dy with an ordinary weight)
    dw[1, 3] = 0.0
    check(dw, dy, x, w, leaves, gates, but=(1, 3))


def test_millions_of_rows_and_leaves():
    """More than a GiB of weighted gradients for 128 outputs.  Whole numbers from -2 to 2, and gates that take two values each: partial sums
    are multiples of 2^-9 and, of 360,000 terms of either sign, far below 2^15, so all are exact but for the last rounding."""
    n, k, n_leaves, d_in, d_out = 270_000, 8, 6, 24, 136
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randint(-2, 3, (n, c), generator=g).to(torch.bfloat16).cuda() for c in (d_in, d_out))
    leaves = torch.randint(0, n_leaves, (n, k), generator=g, dtype=torch.int32).cuda()
    gates = (1 + torch.randint(0, 2, (n, k), generator=g) * 2.0 ** -9).cuda()
    w = torch.zeros(n_leaves, d_out, d_in, dtype=torch.bfloat16).cuda()
    _, dw, db, _ = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("weight", "bias"))
    want, _ = ref.mixture_grad(dy, x, w, None, leaves, gates)
    assert float(want[1].abs().max()) < 2.0 ** 14
    for got, e in ((dw, want[1]), (db, want[2])):
        assert bool(((got.double() - e).abs() <= torch.finfo(got.dtype).eps / 2 * e.abs()).all())
