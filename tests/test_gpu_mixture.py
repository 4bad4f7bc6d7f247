"""Rows that several leaves answer, on the GPU, against the definition in 64 bits.

u = 2^-24, half = half a step of the element type.  y: sums of d_in + 1 terms in f32, weighed and added up over k slots, rounded once:
(d_in + k + 3) u of the terms' magnitudes and half of the result; bf16 with k > 1: the terms of the last sum are held with 11 bits,
half a step of which is 2^-11 of each (and 2^-25 of the unit of the least, which is at most 2^-14 of the largest of the row's: 2^-39
of that).  dx the same with d_out.  dweight, dbias: gates * dy is rounded to
the type (half of each term, after u of the product), summed over up to n positions: half + (n + 2) u of the magnitudes, and the
result's half.  dgates: a sum of d_out inside one of d_in + d_out: (d_in + 2 d_out + 4) u of the magnitudes."""
import math

import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def rows(n, cols, dtype, g, pad=0, scale=1.0):
    buf = torch.full((n, cols + pad), math.nan, dtype=DTYPES[dtype]).cuda()
    buf[:, :cols] = (torch.randn(n, cols, generator=g) * scale).to(DTYPES[dtype]).cuda()
    return buf[:, :cols]


def made(n, k, n_leaves, d_in, d_out, dtype, seed, pad=0, skew=1.0, outside=0.05):
    g = torch.Generator().manual_seed(seed)
    x, dy = rows(n, d_in, dtype, g, pad), rows(n, d_out, dtype, g, pad)
    w = (torch.randn(n_leaves, d_out, d_in, generator=g) * d_in ** -0.5).to(DTYPES[dtype]).cuda()
    b = torch.randn(n_leaves, d_out, generator=g).to(DTYPES[dtype]).cuda()
    liked = torch.softmax(skew * torch.randn(n_leaves, generator=g), 0)
    leaves = torch.multinomial(liked, n * k, replacement=True, generator=g).view(n, k).to(torch.int32)
    leaves[torch.rand(n, k, generator=g) < outside] = -1
    leaves[torch.rand(n, k, generator=g) < outside] = n_leaves
    leaves = leaves.cuda()
    gates = torch.randn(n, k, generator=g).cuda()
    # the weight of a slot without a leaf counts for nothing
    gates = torch.where((leaves < 0) | (leaves >= n_leaves), math.nan, gates)
    return x, dy, w, b, leaves, gates


def held(x, k, mag):
    """What the roundings of a row's terms add, for bf16."""
    if x.dtype == torch.float32 or k == 1:
        return 0.0
    return 2.0 ** -11 * mag + 2.0 ** -39 * mag.amax(1, keepdim=True)


def check_y(y, x, w, b, leaves, gates, what=""):
    want, mag = ref.mixture(x, w, b, leaves, gates)
    half = torch.finfo(x.dtype).eps / 2
    bad = (y.double() - want).abs() > (w.shape[2] + leaves.shape[1] + 3) * U * mag + half * want.abs() + held(x, leaves.shape[1], mag)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def check_grad(got, dy, x, w, b, leaves, gates):
    want, mag = ref.mixture_grad(dy, x, w, b, leaves, gates)
    n_leaves, d_out, d_in = w.shape
    n, k = leaves.shape
    half = torch.finfo(x.dtype).eps / 2
    tols = [(d_out + k + 3) * U, half + (n * k + 2) * U, half + (n * k + 2) * U, (d_in + 2 * d_out + 4) * U]
    halves = [half, half, half, 0.0]
    for name, a, e, m, t, h in zip(("dx", "dweight", "dbias", "dgates"), got, want, mag, tols, halves):
        if a is None:
            continue
        bad = (a.double() - e).abs() > t * m + h * e.abs() + (held(x, max(k, 2), m) if name == "dx" else 0.0)
        assert not bool(bad.any()) and not bool(torch.isnan(a).any()), (name, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


SIZES = [  # n, k, leaves, d_in, d_out, pad
    (1, 1, 1, 1, 1, 0), (1, 4, 255, 700, 256, 0), (3, 2, 5, 137, 33, 0), (4, 9, 31, 64, 1000, 0), (5, 3, 4, 3, 2, 1), (64, 4, 64, 128, 96, 0),
    (200, 1, 7, 40, 24, 8), (333, 3, 13, 137, 33, 6), (1000, 2, 8, 256, 130, 0), (777, 8, 255, 72, 64, 0), (130, 64, 10, 16, 16, 0),
    (2500, 2, 3, 64, 257, 7), (600, 5, 1, 512, 20, 0), (400, 2, 5000, 16, 8, 0), (5000, 2, 1100, 24, 8, 0), (9000, 1, 2, 8, 300, 0), (700, 6, 40, 1000, 4, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(dtype, size):
    n, k, n_leaves, d_in, d_out, pad = size
    x, dy, w, b, leaves, gates = made(n, k, n_leaves, d_in, d_out, dtype, seed=n + d_in, pad=pad)
    check_y(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), x, w, b, leaves, gates)
    check_y(B.gbdt_mixture_product(x, w, leaves, gates), x, w, None, leaves, gates)
    check_grad(B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b), dy, x, w, b, leaves, gates)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates)
    check_grad(got, dy, x, w, None, leaves, gates)


@pytest.mark.parametrize("dtype,size", [("bf16", (20_000, 4, 16, 256, 512)), ("bf16", (3000, 8, 64, 512, 300)), ("f32", (6000, 3, 20, 200, 130)),
                                        ("bf16", (40_000, 2, 9, 64, 48)), ("bf16", (40_000, 2, 7, 64, 100)),
                                        ("bf16", (70_000, 1, 4, 64, 300)), ("bf16", (70_000, 1, 4, 40, 100)), ("f32", (20_000, 1, 4, 40, 100)),
                                        ("bf16", (30_000, 2, 2, 128, 136)), ("f32", (40_000, 2, 3, 24, 20))],
                         ids=str)
def test_larger(dtype, size):
    """Tiles of every kind, lists by many wavefronts, leaves cut into pieces."""
    x, dy, w, b, leaves, gates = made(*size, dtype, seed=1)
    check_y(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), x, w, b, leaves, gates)
    check_grad(B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b), dy, x, w, b, leaves, gates)


def test_several_blocks_of_rows_and_pieces_of_outputs():
    """More slots, and more weighted gradients, than are held at once: 40,000 x 8 x 512 f32 is 655 MB, 20,000 x 4 x 2,000 bf16 320 MB."""
    x, dy, w, b, leaves, gates = made(40_000, 8, 12, 16, 512, "f32", seed=2, outside=0.01)
    check_y(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), x, w, b, leaves, gates)
    x, dy, w, b, leaves, gates = made(20_000, 4, 6, 1024, 2000, "bf16", seed=3, outside=0.01)
    check_grad(B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b), dy, x, w, b, leaves, gates)


@pytest.mark.parametrize("dtype,d_in", [("bf16", 2000), ("bf16", 1999), ("f32", 1000)])
def test_pieces_longer_than_a_listing(dtype, d_in):
    """Sums of 1,500 x d_in matrices that would pass the scratch with short pieces: 120,000 positions of two leaves."""
    x, dy, w, b, leaves, gates = made(40_000, 3, 2, d_in, 1500, dtype, seed=15, outside=0.01)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, want=("weight", "bias"))
    check_grad(got, dy, x, w, b, leaves, gates)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("want", [("x",), ("weight",), ("bias",), ("gates",), ("weight", "bias"), ("x", "gates"), ()], ids=str)
@pytest.mark.parametrize("k", [3, 11])
def test_some_gradients(dtype, want, k):
    x, dy, w, b, leaves, gates = made(300, k, 9, 136, 40, dtype, seed=6)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, want=want)
    assert [g is not None for g in got] == [name in want for name in ("x", "weight", "bias", "gates")]
    check_grad(got, dy, x, w, b, leaves, gates)
    assert B.gbdt_mixture_product_grad(dy[:0], x[:0], w, leaves[:0], gates[:0])[1].abs().sum() == 0


def test_rows_without_a_leaf_and_leaves_without_a_row():
    for n in (3, 500):
        x, dy, w, b, leaves, gates = made(n, 4, 20, 48, 24, "bf16", seed=7)
        leaves[:2] = -1
        leaves[leaves == 5] = 6
        x[1] = math.nan
        x[0] = math.inf
        y = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
        assert bool((y[:2] == 0).all())
        dx, dw, db, dg = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b)
        assert bool((dx[:2] == 0).all()) and bool((dg[:2] == 0).all()) and bool((dw[5] == 0).all()) and bool((db[5] == 0).all())
        check_grad((dx, dw, db, dg), dy, torch.where(leaves[:, :1] * 0 + torch.arange(n).cuda()[:, None] < 2, 0.0, x.float()).to(x.dtype), w, b,
                   leaves, gates)
        leaves[:] = -1
        assert bool((B.gbdt_mixture_product(x, w, leaves, gates, bias=b) == 0).all())
        dx, dw, db, dg = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b)
        assert all(bool((v == 0).all()) for v in (dx, dw, db, dg))


def test_an_infinity_or_nan_stays_in_its_row():
    for n in (3, 400):
        x, dy, w, b, leaves, gates = made(n, 3, 6, 40, 40, "f32", seed=9, outside=0.0)
        clean = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
        x[2, 5] = math.nan
        y = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
        assert bool(torch.isnan(y[2]).all())
        others = torch.arange(n).cuda() != 2
        assert torch.equal(y[others], clean[others])


def test_same_bits_and_rows_behind():
    x, dy, w, b, leaves, gates = made(4000, 4, 30, 96, 80, "bf16", seed=10)
    y = torch.full((4003, 96), 9.0, dtype=torch.bfloat16).cuda()
    one = B.gbdt_mixture_product(x, w, leaves, gates, bias=b, y_out=y[:4000, 8:88]).clone()
    assert bool((y[4000:] == 9).all()) and bool((y[:, :8] == 9).all()) and bool((y[:, 88:] == 9).all())
    first = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b)
    for _ in range(3):
        assert torch.equal(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), one)
        assert all(torch.equal(a, e) for a, e in zip(B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b), first))


def test_one_leaf_a_row_is_the_leaf_product():
    """k = 1 with weights of 1 gives what gbdt_leaf_product does of the same lists."""
    x, dy, w, b, leaves, gates = made(900, 1, 12, 64, 72, "f32", seed=12, outside=0.0)
    order = torch.sort(leaves[:, 0], stable=True)[1].to(torch.int32)
    offsets = torch.zeros(13, dtype=torch.int64).cuda()
    offsets[1:] = torch.cumsum(torch.bincount(leaves[:, 0].long(), minlength=12), 0)
    y = B.gbdt_mixture_product(x, w, leaves, torch.ones(900, 1).cuda(), bias=b)
    z = B.gbdt_leaf_product(x, w, offsets, row_idx=order, bias=b)
    assert float((y - z).abs().max()) <= 2 * (64 + 3) * U * float(ref.mixture(x, w, b, leaves, torch.ones(900, 1).cuda())[1].max())


def test_gradients_against_differences():
    """Of L = <dy, y>, linear in each of x, weight, bias and gates: a difference over any step is the gradient up to the roundings
    of y, (d_in + k + 4) u of its magnitudes at either end."""
    x, dy, w, b, leaves, gates = made(24, 3, 5, 12, 8, "f32", seed=13, outside=0.0)
    got = B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b)
    g = torch.Generator().manual_seed(14)

    def total(x, w, b, gates):
        y = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
        mag = (ref.mixture(x, w, b, leaves, gates)[1] * dy.double().abs()).sum()
        return float((y.double() * dy.double()).sum()), float(mag) * (12 + 3 + 4) * U
    base = dict(x=x, w=w, b=b, gates=gates)
    for name, grad in zip(("x", "w", "b", "gates"), got):
        step = torch.randn(base[name].shape, generator=g).cuda()
        moved = dict(base, **{name: base[name] + step})
        step = (moved[name].double() - base[name].double())
        (l1, t1), (l0, t0) = total(**moved), total(**base)
        want = float((grad.double() * step).sum())
        grad_tol = float((grad.double().abs() * step.abs()).sum()) * U * 2 + 72 * 2 * U * t0 / (19 * U)
        assert abs((l1 - l0) - want) <= t1 + t0 + grad_tol, name


def test_infinities_and_sizes_within_a_row_of_terms():
    """bf16 terms share a power of two by 64 columns: an infinity or a NaN among them leaves the others as they are, and columns of very
    different size keep their own digits."""
    n, k = 300, 3
    x, dy, w, b, leaves, gates = made(n, k, 4, 64, 128, "bf16", seed=21, outside=0.0)
    size = 2.0 ** torch.randint(-60, 60, (128,), generator=torch.Generator().manual_seed(1)).float().cuda()
    w = (w.float() * size[:, None]).to(torch.bfloat16)
    b = (b.float() * size).to(torch.bfloat16)
    w[1, 3], b[2, 70] = math.inf, math.nan
    y = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
    hit3 = (leaves == 1).any(1)
    hit70 = (leaves == 2).any(1)
    assert torch.equal(~torch.isfinite(y[:, 3]), hit3) and torch.equal(torch.isnan(y[:, 70]), hit70)
    clean_w, clean_b = w.clone(), b.clone()
    clean_w[1, 3], clean_b[2, 70] = 0.0, 0.0
    want, mag = ref.mixture(x, clean_w, clean_b, leaves, gates)
    block = mag.view(n, 2, 64).amax(2, keepdim=True).expand(n, 2, 64).reshape(n, 128)
    tol = (64 + 3 + 3) * U * mag + 2.0 ** -8 * want.abs() + 2.0 ** -11 * mag + 2.0 ** -39 * block
    ok = (y.double() - want).abs() <= tol
    ok[:, 3] |= hit3
    ok[:, 70] |= hit70
    assert bool(ok.all())
