"""Products grouped by leaf and their gradients against the definition in 64 bits.

Bounds.  A sum of K products of values held exactly, in f32 in any order, is off by at most (K + 1) 2^-24 of the sum of
magnitudes (products of f32 are rounded as well: that is the 1; one more for the bias).  A result in bf16, of 8 significant
bits, is rounded to nearest: 2^-8 of itself at most; an f32 result 2^-24."""
import pytest
import torch

from oracle import linear_leaves as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def bound(exact, mag, k, dtype):
    return (k + 3) * 2.0 ** -24 * mag + exact.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) + 1e-37


def close(got, exact, mag, k, what):
    assert got.shape == exact.shape, what
    err = (got.double() - exact).abs()
    over = err - bound(exact, mag, k, got.dtype)
    assert bool(torch.isfinite(got).all()), what
    assert float(over.max()) <= 0.0 if over.numel() else True, (what, float(err.max()))


def make(rows, sizes, d_in, d_out, dtype, pad=0, listed=None, seed=0, idx=True):
    """Leaf sizes need not add up to the rows: the rest of the rows is in no leaf."""
    g = torch.Generator().manual_seed(seed)
    total = sum(sizes)
    assert total <= rows
    order = torch.randperm(rows, generator=g)[:total].to(torch.int32) if idx else None
    offs = torch.zeros(len(sizes) + 1, dtype=torch.int64)
    offs[1:] = torch.cumsum(torch.tensor(sizes), 0)

    def mat(cols):
        buf = torch.randn(rows, cols + pad, generator=g).to(DT[dtype])
        return buf.cuda()[:, pad // 2:pad // 2 + cols]
    x, dy = mat(d_in), mat(d_out)
    w = torch.randn(len(sizes), d_out, d_in, generator=g).to(DT[dtype]).cuda()
    b = torch.randn(len(sizes), d_out, generator=g).to(DT[dtype]).cuda()
    return x, dy, w, b, offs.cuda(), order.cuda() if idx else None


CASES = [
    # rows, sizes, d_in, d_out, pad
    (1, [1], 1, 1, 0),
    (1, [0, 0, 1, 0], 8, 16, 0),
    (3, [1, 0, 2], 7, 17, 3),
    (300, [300], 64, 128, 0),
    (300, [128, 0, 1, 129, 42], 65, 129, 2),
    (777, [5, 250, 0, 0, 511, 1], 137, 33, 6),
    (1000, [400, 0, 300], 24, 5, 0),
    (600, [1] * 500, 28, 1, 0),
    (900, [513, 127, 260], 200, 264, 8),
    (900, [513, 127, 260], 200, 264, 1),
    (2, [2], 2000, 3, 0),
    (64, [30, 34], 129, 1, 0),
    (64, [10, 0, 54], 100, 70, 0),
    (64, [3, 61], 5, 40, 1),
    (2000, [700, 650, 650], 264, 200, 0),
    (1200, [300, 800, 0, 100], 72, 48, 0),
    (200, [130, 0, 70], 2000, 33, 0),
    (70, [70], 513, 65, 0),
    (150, [100, 50], 1999, 7, 3),
    (90, [90], 5000, 17, 8),
    (33_500, [20_000, 0, 13_400], 264, 264, 8),
    (66_500, [66_000, 100, 0, 400], 72, 96, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d-%d-%d" % (c[0], len(c[1]), c[2], c[3]))
def test_product_and_gradients(case, dtype):
    from paper_1706_08359_amd import binding as B
    rows, sizes, d_in, d_out, pad = case
    x, dy, w, b, offs, idx = make(rows, sizes, d_in, d_out, dtype, pad)
    # rows of no leaf: what they hold is neither read nor written
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[idx.long()] = True
    x[~inside], dy[~inside] = float("nan"), float("inf")
    y0 = torch.full((rows, d_out + pad), 7.0, dtype=DT[dtype], device="cuda")[:, :d_out]
    y = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b, y_out=y0.clone(memory_format=torch.preserve_format))
    want, mag = ref.leaf_product(x, w, b, offs, idx, y0)
    close(y, want, mag, d_in, "y")
    dx0 = torch.full((rows, d_in), -3.0, dtype=DT[dtype], device="cuda")
    got = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, dx_out=dx0.clone())
    want, mags = ref.leaf_product_grad(dy, x, w, offs, idx, dx0)
    for name, a, e, m, k in zip(("dx", "dw", "db"), got, want, mags, (d_out, max(sizes), max(sizes))):
        close(a, e, m, k, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[5000], [511, 1, 512, 0, 513, 2, 1500, 100, 0, 700], [1023, 0, 1, 4000, 0, 0, 12],
                                   [0, 3000, 0, 3000, 0]], ids=str)
def test_long_leaves_are_summed_in_parts(sizes, dtype):
    from paper_1706_08359_amd import binding as B
    rows = sum(sizes) + 9
    for d_in, d_out in ((40, 24), (13, 3)):
        x, dy, w, b, offs, idx = make(rows, sizes, d_in, d_out, dtype, seed=3)
        got = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight", "bias"))
        again = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight", "bias"))
        assert got[0] is None
        want, mags = ref.leaf_product_grad(dy, x, w, offs, idx, torch.zeros_like(x))
        for name, i in (("dw", 1), ("db", 2)):
            close(got[i], want[i], mags[i], max(sizes), name)
            assert torch.equal(got[i], again[i])
        only = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("bias",))
        assert only[1] is None and torch.equal(only[2], got[2])
        only = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight",))
        assert only[2] is None and torch.equal(only[1], got[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_in, d_out", [(40, 24), (13, 3), (8192, 1024)])
def test_outputs_sums_alone_need_no_inputs(d_in, d_out, dtype):
    """x and weight null, in a workspace of the size that is said to suffice."""
    from paper_1706_08359_amd import binding as B
    sizes = [700, 0, 1, 2000]
    x, dy, w, b, offs, idx = make(2710, sizes, 1, d_out, dtype, seed=6)
    want, mags = ref.leaf_product_grad(dy, x, w, offs, idx, torch.zeros_like(x))
    got = torch.full((len(sizes), d_out), 7.0, dtype=DT[dtype], device="cuda")
    ws = torch.empty(B.gbdt_leaf_product_grad_workspace_bytes(2701, d_in, d_out), dtype=torch.uint8, device="cuda")
    B.gbdt_set_workspace(ws)
    try:
        rc = B.load().gbdt_leaf_product_grad(dy.data_ptr(), d_out, None, 0, None, idx.data_ptr(), offs.data_ptr(), 2701, len(sizes),
                                             2710, d_in, d_out, B.DTYPES[DT[dtype]], None, 0, None, got.data_ptr(),
                                             torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()
    finally:
        B.gbdt_set_workspace(None)
    close(got, want[2], mags[2], max(sizes), "db")


def test_pieces_longer_than_a_copy_of_their_list():
    """So much work a position that pieces are thousands of positions long."""
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(70_100, [62_000, 0, 100, 8000], 2000, 200, "bf16", seed=4)
    got = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("weight", "bias"))
    want, mags = ref.leaf_product_grad(dy, x, w, offs, idx, torch.zeros(70_100, 1, device="cuda").expand(70_100, 2000))
    for i in (1, 2):
        close(got[i], want[i], mags[i], 62_000, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lists_that_are_odd(dtype):
    """No list, offsets that leave out the ends of it or pass them, row ids outside the matrix, no positions at all."""
    from paper_1706_08359_amd import binding as B
    rows, d_in, d_out = 500, 48, 40
    x, dy, w, b, _, idx = make(rows, [100, 200, 150], d_in, d_out, dtype, seed=5)
    bad = idx.clone()
    bad[::17] = -1
    bad[5::23] = rows
    for list_, offs in ((None, [0, 100, 300, 500]), (None, [3, 3, 7, 400]), (idx, [10, 100, 300, 440]),
                        (idx, [-5, 100, 300, 10 ** 12]), (bad, [0, 100, 300, 450]), (idx, [0, 0, 0, 0]),
                        (idx, [450, 450, 450, 450]), (idx[:0], [0, 0, 0, 0])):
        offs = torch.tensor(offs, dtype=torch.int64, device="cuda")
        y0 = torch.full((rows, d_out), 2.0, dtype=DT[dtype], device="cuda")
        y = B.gbdt_leaf_product(x, w, offs, row_idx=list_, bias=None, y_out=y0.clone())
        want, mag = ref.leaf_product(x, w, None, offs, list_, y0)
        close(y, want, mag, d_in, ("y", offs))
        dx0 = torch.full((rows, d_in), 2.0, dtype=DT[dtype], device="cuda")
        got = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=list_, dx_out=dx0.clone())
        want, mags = ref.leaf_product_grad(dy, x, w, offs, list_, dx0)
        for a, e, m in zip(got, want, mags):
            close(a, e, m, 500, offs)
    made = B.gbdt_leaf_product(x, w, torch.tensor([0, 0, 5, 5], device="cuda"), row_idx=idx)
    assert int((made != 0).any(1).sum()) == 5


def test_infinities_and_nan_stay_in_their_row_and_leaf():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(256, [100, 0, 156], 64, 64, "bf16", seed=6)
    clean = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)
    grads = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    r = int(idx[40])
    x2, dy2 = x.clone(), dy.clone()
    x2[r, 3], dy2[r, 5] = float("nan"), float("inf")
    y = B.gbdt_leaf_product(x2, w, offs, row_idx=idx, bias=b)
    assert bool(y[r].isnan().all())
    keep = torch.arange(256, device="cuda") != r
    assert torch.equal(y[keep], clean[keep])
    dx, dw, db = B.gbdt_leaf_product_grad(dy2, x2, w, offs, row_idx=idx)
    assert torch.equal(dx[keep], grads[0][keep]) and not bool(dx[r].isfinite().any())
    assert torch.equal(dw[1:], grads[1][1:]) and torch.equal(db[1:], grads[2][1:])
    assert bool(dw[0, :, 3].isnan().all()) and not bool(dw[0, 5].isfinite().any()) and bool(db[0, 5].isinf())
    rest = torch.ones(64, 64, dtype=torch.bool, device="cuda")
    rest[5], rest[:, 3] = False, False
    assert torch.equal(dw[0][rest], grads[1][0][rest])


def test_rows_past_32_bit_offsets():
    """A matrix of more than 2^31 elements, of which the last rows are used."""
    from paper_1706_08359_amd import binding as B
    rows, d_in = 1_100_000, 2000
    x = torch.empty(rows, d_in, dtype=torch.bfloat16, device="cuda")
    last = torch.arange(rows - 70, rows, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(8)
    x[rows - 70:] = torch.randn(70, d_in, generator=g).bfloat16().cuda()
    w = torch.randn(2, 24, d_in, generator=g).bfloat16().cuda()
    dy = torch.randn(70, 24, generator=g).bfloat16().cuda()
    offs = torch.tensor([0, 33, 70], device="cuda")
    y = B.gbdt_leaf_product(x, w, offs, row_idx=last)
    small = torch.arange(70, dtype=torch.int32, device="cuda")
    want, mag = ref.leaf_product(x[rows - 70:], w, None, offs, small, torch.zeros(70, 24, dtype=torch.bfloat16, device="cuda"))
    close(y[rows - 70:], want, mag, d_in, "y")
    dyl = torch.zeros(rows, 24, dtype=torch.bfloat16, device="cuda")
    dyl[rows - 70:] = dy
    dx0 = torch.zeros(70, d_in, dtype=torch.bfloat16, device="cuda")
    dx = torch.empty(rows, d_in, dtype=torch.bfloat16, device="cuda")
    got = B.gbdt_leaf_product_grad(dyl, x, w, offs, row_idx=last, dx_out=dx)
    want, mags = ref.leaf_product_grad(dy, x[rows - 70:], w, offs, small, dx0)
    close(got[0][rows - 70:], want[0], mags[0], 24, "dx")
    close(got[1], want[1], mags[1], 70, "dw")


def test_gradients_against_differences():
    """<gradient, u> of sum(dy * y) against a central difference of the 64-bit definition, which is linear in x, in the
    weights and in the bias: the difference is exact up to 64-bit rounding, whatever the step."""
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(400, [150, 0, 90, 160], 37, 21, "f32", seed=9)
    dx, dw, db = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    zero = torch.zeros(400, 21, device="cuda")

    def f(x_, w_, b_):
        return float((ref.leaf_product(x_, w_, b_, offs, idx, zero)[0] * dy.double()).sum())
    g = torch.Generator().manual_seed(1)
    x64, w64, b64 = x.double(), w.double(), b.double()
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64).cuda()
        plus, minus = [x64, w64, b64], [x64, w64, b64]
        plus[which], minus[which] = plus[which] + 0.5 * u, minus[which] - 0.5 * u
        slope = f(*plus) - f(*minus)
        got = float((grad.double() * u).sum())
        # every element is off by at most 400 * 2^-24 of its sum of magnitudes (see above); |u| < 5
        _, mags = ref.leaf_product_grad(dy, x, w, offs, idx, torch.zeros_like(x))
        assert abs(got - slope) <= 403 * 2.0 ** -24 * float((mags[which] * u.abs()).sum()) + 1e-9 * abs(slope)


def test_other_stream_workspace_and_graph():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(3000, [2500, 20, 480], 72, 40, "bf16", seed=11)
    y = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)
    grads = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    need = B.gbdt_leaf_product_grad_workspace_bytes(3000, 72, 40)
    own = torch.empty(need, dtype=torch.uint8, device="cuda")
    try:
        B.gbdt_set_workspace(own)
        with torch.cuda.stream(side):
            y2 = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)
            g2 = B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
        side.synchronize()
        assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(grads, g2))
        small = torch.empty(need - 256, dtype=torch.uint8, device="cuda")
        B.gbdt_set_workspace(small)
        with pytest.raises(B.GbdtError, match="workspace"):
            B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)
    finally:
        B.gbdt_set_workspace(None)
    yg, dxg = torch.zeros_like(y), torch.zeros_like(x)
    dwg, dbg = torch.zeros_like(w), torch.zeros_like(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b, y_out=yg)
        B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, dx_out=dxg, dweight_out=dwg, dbias_out=dbg)
    for turn in range(3):
        x.copy_(x.flip(0))
        for t in (yg, dxg, dwg, dbg):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yg, B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)), turn
        for a, e in zip((dxg, dwg, dbg), B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx)):
            assert torch.equal(a, e), turn


def test_the_binding_refuses():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(64, [30, 34], 16, 8, "f32")
    y = torch.zeros(64, 8, device="cuda")
    for bad in (lambda: B.gbdt_leaf_product(x.half(), w.half(), offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x, w.bfloat16(), offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x[:, :15], w, offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x.cpu(), w, offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x[:1].expand(64, 16), w, offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(torch.randn(16, 64, device="cuda").t(), w, offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x, w.transpose(1, 2), offs, row_idx=idx),
                lambda: B.gbdt_leaf_product(x, w, offs.int(), row_idx=idx),
                lambda: B.gbdt_leaf_product(x, w, offs, row_idx=idx.long()),
                lambda: B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b[:, :4]),
                lambda: B.gbdt_leaf_product(x, w, offs, row_idx=idx, y_out=y[:32]),
                lambda: B.gbdt_leaf_product_grad(y[:, :1].expand(64, 8), x, w, offs, row_idx=idx),
                lambda: B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, dweight_out=w[:1])):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: B.gbdt_leaf_product(x, w, offs[:2], row_idx=idx),
                lambda: B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, want=("y",))):
        with pytest.raises(B.GbdtError):
            bad()
