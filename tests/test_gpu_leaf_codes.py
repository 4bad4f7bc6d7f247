"""Rows as 8-bit codes and leaf products of codes, on the GPU, against the definition.

Codes and scales are equal.  A product of codes is exact up to its conversion to f32 (2^-24), two products with scales and the sum with
the bias: 4 u of the magnitudes, and half a step of the result's type; a mixture adds k + 1 u, and for bf16 with k > 1 the 11 bits that
its terms are held with: 2^-11 of each, and 2^-39 of the largest of the row's."""
import math

import pytest
import torch

from oracle import linear_leaves as one_leaf
from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,cols,pad", [(1, 1, 0), (3, 7, 1), (5, 16, 0), (70, 28, 0), (33, 137, 6), (20, 512, 0), (9, 513, 2), (10, 700, 0),
                                        (5, 1024, 0), (4, 1025, 1), (6, 2000, 0), (3, 2049, 0), (2, 9001, 3), (3000, 64, 0)])
def test_codes(dtype, n, cols, pad):
    g = torch.Generator().manual_seed(n + cols)
    buf = torch.full((n, cols + pad), math.inf, dtype=DTYPES[dtype])
    x = torch.randn(n, cols, generator=g) * torch.exp(3 * torch.randn(n, 1, generator=g))
    buf[:, :cols] = x.to(DTYPES[dtype])
    x = buf.cuda()[:, :cols]
    codes, scales = B.gbdt_rows_quantize(x)
    want, want_scales = ref.quantize(x)
    assert codes.shape == (n, B.code_columns(cols)) and torch.equal(scales, want_scales)
    assert torch.equal(codes[:, :cols], want) and bool((codes[:, cols:] == 0).all())
    out = torch.full((n + 1, B.code_columns(cols) + 16), 99, dtype=torch.int8).cuda()
    B.gbdt_rows_quantize(x, codes_out=out[:n, :B.code_columns(cols)])
    assert torch.equal(out[:n, :-16], codes) and bool((out[:n, -16:] == 99).all()) and bool((out[n] == 99).all())


def test_codes_next_to_a_half():
    """Quotients at, just below and just above every half, for scales of all kinds of last places."""
    g = torch.Generator().manual_seed(0)
    out = []
    for top in (127.0, 1.0, 3.14159, 1e-30, 2.7e37, 1.1754944e-36):
        s = float(ref.quantize(torch.tensor([[top]]))[1])
        half = (torch.arange(0, 127).double() + 0.5) * s
        near = half.float()
        row = torch.cat([near, torch.nextafter(near, torch.tensor(math.inf)), torch.nextafter(near, torch.tensor(0.0)),
                         torch.tensor([top])])
        out += [row, -row, row[torch.randperm(row.numel(), generator=g)]]
    x = torch.stack(out).float().cuda()
    codes, scales = B.gbdt_rows_quantize(x)
    want, want_scales = ref.quantize(x)
    assert torch.equal(scales, want_scales) and torch.equal(codes[:, :x.shape[1]], want)


@pytest.mark.parametrize("cols", [24, 600, 3000])
def test_codes_of_rows_that_are_not_finite_or_tiny(cols):
    x = torch.randn(8, cols, generator=torch.Generator().manual_seed(1))
    x[0, cols - 1] = math.nan
    x[1, 0] = math.inf
    x[2, 3] = -math.inf
    x[3] = 0.0
    x[4] *= 1e-42
    x[5] = -0.0
    x[6] = 3.4e38 * torch.sign(x[6])
    codes, scales = B.gbdt_rows_quantize(x.cuda())
    want, want_scales = ref.quantize(x)
    assert torch.equal(codes[:, :cols].cpu(), want)
    assert torch.equal(torch.isnan(scales).cpu(), torch.isnan(want_scales)) and bool((scales[3:6] == 0).all())
    assert torch.equal(scales[6:].cpu(), want_scales[6:])


def made(n, n_leaves, d_in, d_out, seed, extreme=False):
    g = torch.Generator().manual_seed(seed)
    if extreme:
        codes = torch.where(torch.rand(n, d_in, generator=g) < 0.5, -127, 127).to(torch.int8)
        w = torch.where(torch.rand(n_leaves * d_out, d_in, generator=g) < 0.9, codes[0], -codes[0]).to(torch.int8)
    else:
        codes = torch.randint(-127, 128, (n, d_in), generator=g).to(torch.int8)
        w = torch.randint(-127, 128, (n_leaves * d_out, d_in), generator=g).to(torch.int8)
    scales = torch.rand(n, generator=g) + 0.01
    ws = torch.rand(n_leaves, d_out, generator=g) * 0.01
    b = torch.randn(n_leaves, d_out, generator=g)
    w = ref.padded(w).view(n_leaves, d_out, -1)
    return ref.padded(codes).cuda(), scales.cuda(), w.cuda(), ws.cuda(), b.cuda(), g


def values(codes, scales):
    return codes.double() * scales.double()[..., None]


def close(y, want, mag, roundings, k=1):
    half = torch.finfo(y.dtype).eps / 2 if y.dtype != torch.float32 else 0.0
    held = 2.0 ** -11 * mag + 2.0 ** -39 * mag.amax(1, keepdim=True) if half and k > 1 else 0.0
    return bool(((y.double() - want).abs() <= (roundings + 1) * U * mag + half * want.abs() + held).all())


SIZES = [(1, 255, 700, 256), (3, 4, 1, 1), (9, 5, 28, 16), (40, 3, 137, 33), (64, 64, 128, 100), (500, 7, 64, 10), (1000, 31, 2000, 64),
         (3000, 5, 200, 130), (20_000, 8, 144, 300), (70_000, 4, 40, 24), (60_000, 3, 272, 128), (40_000, 2, 128, 512), (70_000, 5, 100, 120)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_leaf_products(dtype, size):
    n, n_leaves, d_in, d_out = size
    codes, scales, w, ws, b, g = made(*size, seed=n)
    idx = torch.randperm(n, generator=g).to(torch.int32)
    idx[torch.rand(n, generator=g) < 0.02] = -1
    idx[torch.rand(n, generator=g) < 0.02] = n
    offs = torch.sort(torch.cat([torch.randint(0, n + 1, (n_leaves,), generator=g), torch.tensor([n])]))[0].cuda()
    idx = idx.cuda()
    y0 = torch.full((n, d_out), 3.0, dtype=DTYPES[dtype]).cuda()
    y = B.gbdt_leaf_product_codes(codes, scales, w, ws, offs, row_idx=idx, bias=b, dtype=DTYPES[dtype], y_out=y0.clone())
    want, mag = one_leaf.leaf_product(values(codes, scales), values(w, ws), b, offs, idx, y0)
    assert close(y, want, mag, 4)
    plain = B.gbdt_leaf_product_codes(codes, scales, w, ws, offs, dtype=DTYPES[dtype])
    want, mag = one_leaf.leaf_product(values(codes, scales), values(w, ws), None, offs, None, torch.zeros_like(y0))
    assert close(plain, want, mag, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 3, 9])
@pytest.mark.parametrize("size", [(1, 255, 700, 256), (5, 4, 20, 3), (64, 64, 128, 96), (900, 13, 137, 33), (5000, 6, 256, 200),
                                  (12_000, 5, 64, 600), (30_000, 5, 64, 100), (70_000, 4, 48, 300)], ids=str)
def test_mixtures(dtype, k, size):
    n, n_leaves, d_in, d_out = size
    codes, scales, w, ws, b, g = made(*size, seed=n + k)
    leaves = torch.randint(-1, n_leaves + 1, (n, k), generator=g, dtype=torch.int32).cuda()
    gates = torch.randn(n, k, generator=g).cuda()
    y = B.gbdt_mixture_product_codes(codes, scales, w, ws, leaves, gates, bias=b, dtype=DTYPES[dtype])
    want, mag = ref.mixture(values(codes, scales), values(w, ws), b, leaves, gates)
    assert close(y, want, mag, 5 + k, k)
    y = B.gbdt_mixture_product_codes(codes, scales, w, ws, leaves, gates, dtype=DTYPES[dtype])
    want, mag = ref.mixture(values(codes, scales), values(w, ws), None, leaves, gates)
    assert close(y, want, mag, 5 + k, k)


@pytest.mark.parametrize("n", [2, 300])
def test_the_largest_sums(n):
    """131,072 products of 127 x 127, of one sign: the sum's last bit before it would leave 32 bits."""
    codes, scales, w, ws, b, g = made(n, 2, 131_072, 3, seed=3, extreme=True)
    codes[1] = 127
    w[1] = 127
    leaves = torch.tensor([0, 1], dtype=torch.int32).repeat(n, 1).cuda()
    gates = torch.ones(n, 2).cuda()
    y = B.gbdt_mixture_product_codes(codes, scales, w, ws, leaves, gates)
    want, mag = ref.mixture(values(codes, scales), values(w, ws), None, leaves, gates)
    assert close(y, want, mag, 7)


def test_a_row_without_a_scale():
    x = torch.randn(300, 40, generator=torch.Generator().manual_seed(5)).cuda()
    x[7, 3] = math.nan
    codes, scales = B.gbdt_rows_quantize(x)
    _, _, w, ws, b, _ = made(1, 3, 40, 8, seed=6)
    leaves = torch.zeros(300, 1, dtype=torch.int32).cuda()
    leaves[9] = -1
    x[9, 0] = math.nan
    y = B.gbdt_mixture_product_codes(codes, scales, w, ws, leaves, torch.ones(300, 1).cuda(), bias=b)
    assert bool(torch.isnan(y[7]).all()) and bool((y[9] == 0).all())
    assert not bool(torch.isnan(y[torch.arange(300).cuda() != 7]).any())


@pytest.mark.parametrize("n,d_out", [(70_000, 200), (60_000, 300), (300, 64)])
def test_offsets_past_the_list_and_leaves_before_the_first(n, d_out):
    """Offsets outside the list are its ends, positions before the first and from the last on belong to no leaf."""
    codes, scales, w, ws, b, g = made(n, 4, 64, d_out, seed=n)
    offs = torch.tensor([n // 10, n // 2, n // 2, n - n // 7, n + 50]).cuda()
    y = B.gbdt_leaf_product_codes(codes, scales, w, ws, offs, bias=b, y_out=torch.full((n, d_out), 3.0).cuda())
    want, mag = one_leaf.leaf_product(values(codes, scales), values(w, ws), b, offs, None, torch.full((n, d_out), 3.0).cuda())
    assert close(y, want, mag, 4) and bool((y[:n // 10] == 3).all())
