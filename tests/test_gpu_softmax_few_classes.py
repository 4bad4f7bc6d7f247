"""bf16 gradients of a softmax over few classes, where no element of p - [v = y] stands out of its row or its column.

Up to 128 classes the gradient by the scores meets the operands as the sum of two bf16 values, off by 2^-16 of an element at
most.  Rounding a result to bf16 is off by 1.66e-3 of it, root mean square; what 2^-16 adds, 9e-6 root mean square in every
element independently, is a factor of 1 + 2e-5 of that error, and f32 sums and exponentials, a few 1e-6, add less.  1.01 leaves
room for sums that cancel to a tenth of their terms."""
import pytest
import torch

from oracle import linear_leaves as ref

pytestmark = pytest.mark.gpu


def make(n, v, dim, scale, seed, drawn, ignore=0.1):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn(n, dim, generator=g).bfloat16()
    c = (scale * dim ** -0.5 * torch.randn(v, dim, generator=g)).bfloat16()
    if drawn:  # as a model's own labels are
        y = torch.multinomial(torch.softmax(h.float() @ c.float().t(), 1), 1, generator=g)[:, 0].int()
    else:
        y = torch.randint(0, v, (n,), generator=g, dtype=torch.int32)
    y[torch.rand(n, generator=g) < ignore] = -1
    return h.cuda(), c.cuda(), y.cuda(), (torch.rand(n, generator=g) + 0.25).cuda()


def ratios(h, c, y, w, scale):
    from paper_1706_08359_amd import binding as B
    _, lse = B.gbdt_softmax_loss(h, c, y)
    got = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=scale)
    again = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=scale)
    want, _ = ref.softmax_grad(h, c, y, lse, w, scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    return [float((a.double() - e).norm()) / float((e.bfloat16().double() - e).norm()) for a, e in zip(got, want)]


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("spread", [2.0, 12.0])
@pytest.mark.parametrize("n,v,dim", [(4000, 2, 64), (700, 3, 16), (1500, 10, 40), (260, 50, 137), (3000, 100, 24), (900, 127, 200),
                                     (5000, 128, 8), (70_000, 10, 16)])
def test_error_is_that_of_rounding_the_result(n, v, dim, spread, drawn):
    for what, ratio in zip(("dh", "dc"), ratios(*make(n, v, dim, spread, v, drawn), 1.0 / n)):
        assert ratio <= 1.01, (what, ratio)


@pytest.mark.parametrize("v", [128, 129])
def test_both_sides_of_the_limit_agree(v):
    """The same rows and classes, one class of which has a probability of zero."""
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(600, 128, 48, 2.0, 5, True)
    _, lse = B.gbdt_softmax_loss(h, c, y)
    few = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=0.1)
    if v == 129:
        h, c = torch.nn.functional.pad(h, (0, 8), value=16.0), torch.nn.functional.pad(c, (0, 8))
        c = torch.cat([c, torch.zeros_like(c[:1])])
        c[128, 48:] = -16.0
    got = B.gbdt_softmax_grad(h, c, y, lse, row_weight=w, scale=0.1)
    for a, e in ((got[0][:, :48], few[0]), (got[1][:128, :48], few[1])):
        assert float((a.double() - e.double()).norm()) <= (0.0 if v == 128 else 4e-3) * float(e.double().norm())


def test_no_rows_and_nothing_but_ignored_ones():
    from paper_1706_08359_amd import binding as B
    h, c, y, w = make(300, 30, 48, 2.0, 7, False)
    dh, dc = B.gbdt_softmax_grad(h[:0], c, y[:0], torch.empty(0, device="cuda"))
    assert dh.shape == (0, 48) and dc.shape == (30, 48) and not bool(dc.any())
    y.fill_(30)
    h[::2], w[::3] = float("nan"), float("inf")
    dh, dc = B.gbdt_softmax_grad(h, c, y, torch.zeros(300, device="cuda"), row_weight=w)
    assert not bool(dh.any()) and not bool(dc.any())
