"""The softmax loss over many classes, its gradients and its columns of statistics against the definition in 64 bits.

Bounds.  A score is a sum of dim products in f32: off by at most a = (dim + 1) 2^-24 of its magnitudes.  Exponentials are
taken of (s - base) log2 e: the difference and the product each add 2^-24 of their size, the base-2 exponential 2^-23, so an
exponential of |s - base| <= D is off by e = a + 4 D 2^-24 + 2^-22 of itself.  lse is off by that plus the rounding of a sum of
n_classes terms and of the final sum and logarithm; a probability by the sum of both.  G is rounded to the operands' type
(bf16 keeps 8 significant bits: 2^-8 of each element at most) before its products, whose f32 sums and final rounding are as in
any product."""
import pytest
import torch

from oracle import linear_leaves as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def make(n, v, dim, dtype, seed=0, scale=2.0, pad=0, ignore=0.2):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn(n, dim + pad, generator=g).to(DT[dtype]).cuda()[:, pad // 2:pad // 2 + dim]
    c = (scale * dim ** -0.5 * torch.randn(v, dim + pad, generator=g)).to(DT[dtype]).cuda()[:, pad // 2:pad // 2 + dim]
    y = torch.randint(0, v, (n,), generator=g, dtype=torch.int32)
    out = torch.rand(n, generator=g)
    y[out < ignore / 2] = -1
    y[(out >= ignore / 2) & (out < ignore)] = v
    w = torch.rand(n, generator=g) + 0.25
    return h, c, y.cuda(), w.cuda()


def exp_error(h, c, base):
    """Bound on the relative error of exp(s - base): [n, v]."""
    s, mag = ref.scores(h, c)
    return (h.shape[1] + 1) * U * mag + 4 * (s - base[:, None]).abs() * U + 4 * U


def within(got, want, bound, what):
    assert got.shape == want.shape, what
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), (what, float(err.max()), float((err - bound).max()))


def check_loss(B, h, c, y):
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    want_loss, want_lse = ref.softmax_loss(h, c, y)
    use = ref.counted(y, h.shape[0], c.shape[0], h.device)
    s, mag = ref.scores(h, c)
    top = s.max(1)[0]
    # the sum's terms, weighted by their probabilities, are at most as far off as the furthest that matters: use the maximum
    # over classes of p * error, summed; then n_classes roundings of partial sums (all terms positive) and the logarithm's
    p = torch.exp(s - torch.logsumexp(s, 1)[:, None])
    rel = (p * exp_error(h, c, top)).sum(1) + (c.shape[0] / 16 + 64) * U
    b_lse = rel + 4 * U * (torch.logsumexp(s, 1).abs() + top.abs() + 1.0)
    zero = torch.zeros_like(b_lse)
    within(lse, want_lse, torch.where(use, b_lse, zero), "lse")
    pick_mag = mag.max(1)[0] * (h.shape[1] + 1) * U
    if y is not None:
        within(loss, want_loss, torch.where(use, b_lse + pick_mag + 2 * U * want_loss.abs(), zero), "loss")
    else:
        assert loss is None
    return loss, lse


def check_grad(B, h, c, y, w, scale, lse):
    n, v, dim = h.shape[0], c.shape[0], h.shape[1]
    dh, dc = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=scale)
    (want_dh, want_dc), (mag_h, mag_c) = ref.softmax_grad(h, c, y, lse, w, scale)
    use = ref.counted(y, n, v, h.device)[:, None]
    s, _ = ref.scores(h, c)
    weight = torch.ones(n, device="cuda", dtype=torch.float64) if w is None else w.double().abs()
    p = torch.exp(s - lse.double()[:, None])
    rounding = 2.0 ** -8 if h.dtype == torch.bfloat16 else U
    g = ref.score_gradient(h, c, y, lse, w)
    zero = torch.zeros_like(g)
    g_err = torch.where(use, weight[:, None] * p * exp_error(h, c, lse.double()) + (1.01 * rounding + 2 * U) * g.abs(), zero)
    hs = torch.where(use, h.double(), torch.zeros_like(h, dtype=torch.float64))
    last = 2.0 ** -8 if h.dtype == torch.bfloat16 else 4 * U
    within(dh, want_dh, abs(scale) * (g_err @ c.double().abs()) + (v + 4) * U * mag_h + last * want_dh.abs() + 1e-37, "dh")
    within(dc, want_dc, abs(scale) * (g_err.t().contiguous() @ hs.abs()) + (n + 4) * U * mag_c + last * want_dc.abs() + 1e-37, "dc")
    return dh, dc


def check_stats(B, h, c, y, lse, begin, end):
    grad, hess = B.gbdt_softmax_stats(h, c, y, lse, begin, end)
    want_grad, want_hess = ref.softmax_stats(h, c, y, lse, begin, end)
    use = ref.counted(y, h.shape[0], c.shape[0], h.device)
    s, _ = ref.scores(h, c[begin:end])
    p = torch.exp(s - lse.double()[:, None])
    e = torch.where(use[:, None], p * exp_error(h, c[begin:end], lse.double()), torch.zeros_like(p)).t()
    within(grad, want_grad, e + U * want_grad.abs() + 1e-37, "grad")
    within(hess, want_hess, 2 * e * (1 + e) + e * p.t() + 4 * U * (p.t() + p.t() ** 2) * use + 1e-37, "hess")
    return grad, hess


CASES = [
    # rows, classes, dim, pad
    (1, 1, 1, 0), (1, 2, 8, 0), (1, 1000, 64, 0), (17, 3, 7, 2), (33, 129, 33, 0), (130, 257, 64, 8),
    (129, 1000, 137, 6), (5, 5000, 16, 0), (700, 16, 24, 0), (1500, 10, 40, 0), (260, 515, 200, 0), (300, 300, 513, 1),
    (16, 4099, 512, 0), (20, 700, 8, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d-%d" % c[:3])
def test_loss_gradients_and_stats(case, dtype):
    from paper_1706_08359_amd import binding as B
    n, v, dim, pad = case
    h, c, y, w = make(n, v, dim, dtype, pad=pad)
    if n == 1:
        y.zero_()
    _, lse = check_loss(B, h, c, y)
    check_grad(B, h, c, y, w, 1.0 / n, lse)
    check_grad(B, h, c, y, None, -2.0, lse)
    for begin, end in ((0, v), (v // 3, min(v, v // 3 + 1)), (v // 2, min(v, v // 2 + 17)), (v, v)):
        check_stats(B, h, c, y, lse, begin, end)
    # rows without labels: every row counts
    _, lse = check_loss(B, h, c, None)
    p, _ = check_stats(B, h, c, None, lse, 0, v)
    assert float((p.sum(0) - 1).abs().max()) < 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ignored_rows_may_hold_anything(dtype):
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(200, 300, 64, dtype, seed=2)
    ignored = (y < 0) | (y >= 300)
    assert 10 < int(ignored.sum()) < 190
    clean_loss, clean_lse = B.gbdt_softmax_loss(h, c, y)
    clean = B.gbdt_softmax_grad(h, c, y, clean_lse, row_weight=w, scale=0.5)
    clean_stats = B.gbdt_softmax_stats(h, c, y, clean_lse, 7, 90)
    rows = ignored.nonzero()[:, 0]
    for k, value in enumerate((float("nan"), float("inf"), -float("inf"))):
        h[rows[k::3], k] = value
    w[rows] = float("nan")
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    assert torch.equal(loss, clean_loss) and torch.equal(lse, clean_lse)
    assert float(loss[rows].abs().max()) == 0.0 and float(lse[rows].abs().max()) == 0.0
    for a, e in zip(B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=0.5), clean):
        assert torch.equal(a, e)
    assert float(clean[0][rows].abs().max()) == 0.0
    for a, e in zip(B.gbdt_softmax_stats(h, c, y, lse, 7, 90), clean_stats):
        assert torch.equal(a, e)
    # nothing but ignored rows
    y.fill_(-1)
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    dh, dc = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w)
    assert not bool(loss.any()) and not bool(lse.any()) and not bool(dh.any()) and not bool(dc.any())


def test_large_infinite_and_nan_scores():
    from paper_1706_08359_amd import binding as B
    inf = float("inf")
    # scores of +-3e4: only the largest counts, nothing overflows
    h = torch.tensor([[1.0, 0.0], [-1.0, 0.0], [0.0, 1.0]], device="cuda")
    c = torch.tensor([[3e4, 0.0], [-3e4, 0.0], [0.0, 0.0]], device="cuda")
    y = torch.tensor([0, 0, 2], dtype=torch.int32, device="cuda")
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    assert lse[:2].tolist() == [3e4, 3e4] and loss[:2].tolist() == [0.0, 6e4]
    assert abs(float(lse[2]) - 1.0986123) < 1e-6
    dh, dc = B.gbdt_softmax_grad(h, c, y, lse)
    assert dh[0].tolist() == [0.0, 0.0] and dh[1].tolist() == [-6e4, 0.0]
    # whole columns of tiles far below or above the rest, over several tiles
    v = 700
    c = torch.zeros(v, 8, device="cuda")
    c[:, 0] = torch.linspace(-200, 200, v, device="cuda")
    h = torch.zeros(4, 8, device="cuda")
    h[:, 0] = torch.tensor([1.0, -1.0, 10.0, 0.0], device="cuda")
    y = torch.tensor([v - 1, 0, 5, 3], dtype=torch.int32, device="cuda")
    check_loss(B, h, c, y)
    # what the formula gives: an infinite score, all scores -inf, a NaN
    h = torch.tensor([[inf], [1.0], [-inf], [float("nan")]], device="cuda")
    c = torch.tensor([[1.0], [2.0]], device="cuda")
    y = torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda")
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    assert lse[0] == inf and lse[2] == -inf and bool(lse[3].isnan()) and bool(loss[3].isnan())
    assert abs(float(loss[1]) - 0.3132617) < 1e-6
    # one class at -inf beside others is a probability of zero, not a NaN
    c = torch.tensor([[1.0, 0.0], [-inf, 0.0], [0.5, 0.0]], device="cuda")
    h = torch.tensor([[1.0, 1.0]], device="cuda")
    c[:, 1] = 0.25
    loss, lse = B.gbdt_softmax_loss(h, c, torch.zeros(1, dtype=torch.int32, device="cuda"))
    want = torch.logsumexp(torch.tensor([1.25, 0.75], dtype=torch.float64), 0)
    assert abs(float(lse[0]) - float(want)) < 1e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_pieces_of_classes_and_parts_of_rows(dtype):
    """So many rows that a piece holds only some of the classes, and the classes' gradient sums over long columns."""
    from paper_1706_08359_amd import binding as B
    n = 150_000 if dtype == "bf16" else 80_000
    h, c, y, w = make(n, 1300, 8, dtype, seed=4)
    _, lse = check_loss(B, h, c, y)
    first = check_grad(B, h, c, y, w, 1.0 / n, lse)
    again = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n)
    assert all(torch.equal(a, e) for a, e in zip(first, again))
    only = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n, want=("h",))
    assert only[1] is None and torch.equal(only[0], first[0])
    only = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / n, want=("classes",))
    assert only[0] is None and torch.equal(only[1], first[1])


@pytest.mark.parametrize("n,dtype", [(300_000, "bf16"), (160_000, "f32")])
def test_pieces_of_a_few_hundred_classes(n, dtype):
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(n, 1300, 8, dtype, seed=11)
    _, lse = B.gbdt_softmax_loss(h, c, y)
    check_grad(B, h, c, y, w, 1.0 / n, lse)


def test_many_rows_of_few_classes_and_many_dimensions():
    """More rows of a tile's classes in one workgroup's share than it lists at a time."""
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(8000, 10, 8192, "bf16", seed=9, scale=1.0)
    _, lse = check_loss(B, h, c, y)
    first = check_grad(B, h, c, y, w, 1.0 / 8000, lse)
    again = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=1.0 / 8000)
    assert all(torch.equal(a, e) for a, e in zip(first, again))


@pytest.mark.parametrize("n,v,dim", [(1, 3000, 64), (40, 2000, 512), (700, 5000, 256)])
def test_bf16_gradients_are_as_exact_as_their_own_rounding(n, v, dim):
    """Root mean square error below 1.25 times that of the exact results rounded to bf16: among many classes the label's
    element outweighs its row and its column, and it must not be rounded before the product."""
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(n, v, dim, "bf16", seed=10, ignore=0.0)
    _, lse = B.gbdt_softmax_loss(h, c, y)
    got = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=0.3)
    want, _ = ref.softmax_grad(h, c, y, lse, w, 0.3)
    for a, e in zip(got, want):
        err = float((a.double() - e).norm())
        assert err <= 1.25 * float((e.bfloat16().double() - e).norm()), (n, v, dim)


def test_loss_takes_many_rows_in_turns():
    """More maxima and sums than one launch's scratch holds."""
    from paper_1706_08359_amd import binding as B
    n, v = 260_000, 20_000
    h, c, y, _ = make(n, v, 8, "bf16", seed=5)
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    for at in (0, n // 2 - 50, n - 300):
        part_loss, part_lse = check_loss(B, h[at:at + 300], c, y[at:at + 300])
        assert torch.equal(part_loss, loss[at:at + 300]) and torch.equal(part_lse, lse[at:at + 300])


def test_no_rows():
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(4, 30, 16, "f32")
    h, y, w = h[:0], y[:0], w[:0]
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    dh, dc = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w)
    assert loss.numel() == lse.numel() == dh.numel() == 0 and not bool(dc.any())
    grad, hess = B.gbdt_softmax_stats(h, c, y, lse, 0, 30)
    assert grad.shape == hess.shape == (30, 0)


def test_gradients_against_differences():
    """<gradient, u> against a central difference of the 64-bit loss along u: off by the third derivative, below
    (6 |s'|)^3 / 6 eps^2 for scores that move at s' <= 20 a unit, and by the gradient's own bounds (f32 operands)."""
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(60, 90, 24, "f32", seed=6, scale=1.0)
    _, lse = B.gbdt_softmax_loss(h, c, y)
    dh, dc = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=0.125)

    def f(h_, c_):
        loss, _ = ref.softmax_loss(h_, c_, y)
        return float(0.125 * (w.double() * loss).sum())
    g = torch.Generator().manual_seed(2)
    eps = 1e-5
    for grad, which in ((dh, 0), (dc, 1)):
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64).cuda()
        plus, minus = [h.double(), c.double()], [h.double(), c.double()]
        plus[which], minus[which] = plus[which] + eps * u, minus[which] - eps * u
        slope = (f(*plus) - f(*minus)) / (2 * eps)
        got = float((grad.double() * u).sum())
        assert abs(got - slope) <= 1e-5 * float((grad.double() * u).abs().sum()) + 60 * 1.25 * 0.125 * 288000 * eps ** 2


def test_columns_feed_a_histogram():
    """grad[i] and hess[i] are what gbdt_hist_build takes: the bins of a feature sum to the column."""
    from paper_1706_08359_amd import binding as B
    n = 3000
    h, c, y, _ = make(n, 50, 16, "f32", seed=7)
    _, lse = B.gbdt_softmax_loss(h, c, y)
    grad, hess = B.gbdt_softmax_stats(h, c, y, lse, 10, 14)
    bins = torch.randint(0, 64, (n, 5), dtype=torch.uint8, generator=torch.Generator().manual_seed(1)).cuda()
    packed = B.gbdt_bins_pack(bins, 64)
    for i in range(4):
        hist = B.hist_to_numpy(B.gbdt_hist_build(packed, n, 5, 64, None, n, grad[i], hess[i]))
        assert int(hist["count"][0].sum()) == n
        tol = 1e-5 * 64
        assert abs(hist["grad"][2].sum() - float(grad[i].double().sum())) <= tol * float(grad[i].abs().sum())
        assert abs(hist["hess"][4].sum() - float(hess[i].double().sum())) <= tol * float(hess[i].sum())


def test_other_stream_workspace_and_graph():
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(500, 900, 64, "bf16", seed=8)
    loss, lse = B.gbdt_softmax_loss(h, c, y)
    grads = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w)
    stats = B.gbdt_softmax_stats(h, c, y, lse, 3, 40)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    need = B.gbdt_softmax_workspace_bytes(500, 900, 64, torch.bfloat16)
    own = torch.empty(need, dtype=torch.uint8, device="cuda")
    try:
        B.gbdt_set_workspace(own)
        with torch.cuda.stream(side):
            loss2, lse2 = B.gbdt_softmax_loss(h, c, y)
            grads2 = B.gbdt_softmax_grad(h, c, y, lse2, row_weight=w)
        side.synchronize()
        assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
        assert all(torch.equal(p, q) for p, q in zip(grads, grads2))
        B.gbdt_set_workspace(own[:(1 << 18) + 256])
        with pytest.raises(B.GbdtError, match="workspace"):
            B.gbdt_softmax_loss(h, c, y)
    finally:
        B.gbdt_set_workspace(None)
    out = [torch.zeros_like(t) for t in (loss, lse, *grads, *stats)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gbdt_softmax_loss(h, c, y, loss_out=out[0], lse_out=out[1])
        B.gbdt_softmax_grad(h, c, y, out[1], row_weight=w, dh_out=out[2], dclasses_out=out[3])
        B.gbdt_softmax_stats(h, c, y, out[1], 3, 40, grad_out=out[4], hess_out=out[5])
    for turn in range(3):
        h.copy_(h.flip(0))
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        loss, lse = B.gbdt_softmax_loss(h, c, y)
        want = (loss, lse, *B.gbdt_softmax_grad(h, c, y, lse, row_weight=w), *B.gbdt_softmax_stats(h, c, y, lse, 3, 40))
        for a, e in zip(out, want):
            assert torch.equal(a, e), turn


def test_the_binding_refuses():
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(20, 30, 16, "f32")
    lse = torch.zeros(20, device="cuda")
    for bad in (lambda: B.gbdt_softmax_loss(h.half(), c.half(), y), lambda: B.gbdt_softmax_loss(h, c.bfloat16(), y),
                lambda: B.gbdt_softmax_loss(h, c[:, :8], y), lambda: B.gbdt_softmax_loss(h, c, y.long()),
                lambda: B.gbdt_softmax_loss(h, c, y[:10]), lambda: B.gbdt_softmax_loss(h.cpu(), c, y),
                lambda: B.gbdt_softmax_grad(h, c, None, lse), lambda: B.gbdt_softmax_grad(h, c, y, lse[:3]),
                lambda: B.gbdt_softmax_grad(h, c, y, lse.double()),
                lambda: B.gbdt_softmax_grad(h, c, y, lse, row_weight=w[:3]),
                lambda: B.gbdt_softmax_grad(h, c, y, lse, dh_out=h[:1].expand(20, 16)),
                lambda: B.gbdt_softmax_stats(h, c, y, lse, 0, 4, grad_out=torch.zeros(20, 4, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: B.gbdt_softmax_stats(h, c, y, lse, -1, 4), lambda: B.gbdt_softmax_stats(h, c, y, lse, 4, 3),
                lambda: B.gbdt_softmax_stats(h, c, y, lse, 0, 31), lambda: B.gbdt_softmax_grad(h, c, y, lse, want=("y",))):
        with pytest.raises(B.GbdtError):
            bad()
