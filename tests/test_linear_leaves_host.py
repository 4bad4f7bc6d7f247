"""What the linear-leaf and softmax calls refuse, before any GPU work (addresses here are never followed)."""
import pytest
import torch

from oracle import linear_leaves as ref
from paper_1706_08359_amd import binding as B

P, EINVAL, EUNSUPPORTED = 4096, -1, -2


def leaf(x=P, ld_x=8, w=P, bias=P, idx=P, offs=P, pos=10, leaves=2, rows=10, d_in=8, d_out=4, dtype=0, y=P, ld_y=4):
    return B.load().gbdt_leaf_product(x, ld_x, w, bias, idx, offs, pos, leaves, rows, d_in, d_out, dtype, y, ld_y, None)


def leaf_grad(dy=P, ld_dy=4, x=P, ld_x=8, w=P, idx=P, offs=P, pos=10, leaves=2, rows=10, d_in=8, d_out=4, dtype=0, dx=P, ld_dx=8,
              dw=P, db=P):
    return B.load().gbdt_leaf_product_grad(dy, ld_dy, x, ld_x, w, idx, offs, pos, leaves, rows, d_in, d_out, dtype, dx, ld_dx, dw,
                                           db, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(offs=None), dict(y=None), dict(ld_x=7), dict(ld_y=3),
                                 dict(pos=-1), dict(leaves=0), dict(rows=-1), dict(d_in=0), dict(d_out=0), dict(dtype=2),
                                 dict(dtype=-1), dict(idx=None, pos=11), dict(x=P + 2), dict(w=P + 1, dtype=1), dict(y=P + 1, dtype=1),
                                 dict(bias=P + 2), dict(offs=P + 4), dict(idx=P + 2)], ids=str)
def test_leaf_product_refuses(bad):
    assert leaf(**bad) == EINVAL


@pytest.mark.parametrize("big", [dict(pos=1 << 30), dict(rows=1 << 30), dict(leaves=1 << 24), dict(d_in=1 << 24, ld_x=1 << 24),
                                 dict(d_out=1 << 24, ld_y=1 << 24)], ids=str)
def test_leaf_product_limits(big):
    assert leaf(**big) == EUNSUPPORTED


def test_nothing_to_do():
    assert leaf(pos=0, x=None, y=None) == 0
    assert leaf(rows=0, x=None, y=None) == 0
    assert leaf_grad(dx=None, dw=None, db=None) == 0


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(w=None), dict(offs=None), dict(ld_dy=3), dict(ld_x=7), dict(ld_dx=7),
                                 dict(pos=-1), dict(leaves=0), dict(d_in=0), dict(dtype=7), dict(dx=P + 2), dict(dw=P + 1),
                                 dict(db=P + 3), dict(dy=P + 1, dtype=1)], ids=str)
def test_leaf_product_grad_refuses(bad):
    assert leaf_grad(**bad) == EINVAL


def loss(h=P, ld_h=8, c=P, ld_c=8, y=P, n=5, v=7, dim=8, dtype=0, out=P, lse=P):
    return B.load().gbdt_softmax_loss(h, ld_h, c, ld_c, y, n, v, dim, dtype, out, lse, None)


def grad(h=P, ld_h=8, c=P, ld_c=8, y=P, lse=P, w=None, n=5, v=7, dim=8, dtype=0, dh=P, ld_dh=8, dc=P, ld_dc=8):
    return B.load().gbdt_softmax_grad(h, ld_h, c, ld_c, y, lse, w, 1.0, n, v, dim, dtype, dh, ld_dh, dc, ld_dc, None)


def stats(h=P, ld_h=8, c=P, ld_c=8, y=P, lse=P, n=5, v=7, dim=8, dtype=0, a=0, b=7, g=P, k=P, ld=5):
    return B.load().gbdt_softmax_stats(h, ld_h, c, ld_c, y, lse, n, v, dim, dtype, a, b, g, k, ld, None)


COMMON = [dict(h=None), dict(c=None), dict(ld_h=7), dict(ld_c=7), dict(n=-1), dict(v=0), dict(dim=0), dict(dtype=2), dict(h=P + 2),
          dict(c=P + 1, dtype=1)]


@pytest.mark.parametrize("bad", COMMON, ids=str)
def test_softmax_refuses(bad):
    assert loss(**bad) == EINVAL and grad(**bad) == EINVAL and stats(**bad) == EINVAL


@pytest.mark.parametrize("call,bad", [(loss, dict(lse=None)), (loss, dict(y=None)), (loss, dict(out=None)), (grad, dict(y=None)),
                                      (grad, dict(lse=None)), (grad, dict(ld_dh=7)), (grad, dict(ld_dc=7)), (grad, dict(dh=P + 2)),
                                      (grad, dict(dc=P + 1, dtype=1)), (stats, dict(a=-1)), (stats, dict(a=5, b=4)), (stats, dict(b=8)),
                                      (stats, dict(lse=None)), (stats, dict(g=None)), (stats, dict(k=None)), (stats, dict(ld=4))],
                         ids=str)
def test_softmax_refuses_more(call, bad):
    assert call(**bad) == EINVAL


@pytest.mark.parametrize("big", [dict(n=1 << 30), dict(v=1 << 30), dict(dim=1 << 24, ld_h=1 << 24, ld_c=1 << 24)], ids=str)
def test_softmax_limits(big):
    assert loss(**big) == EUNSUPPORTED
    assert grad(ld_dh=1 << 24, ld_dc=1 << 24, **big) == EUNSUPPORTED
    assert stats(ld=1 << 30, **big) == EUNSUPPORTED


def test_softmax_nothing_to_do():
    assert loss(n=0, h=None, y=None, out=None, lse=None) == 0
    assert grad(dh=None, dc=None) == 0
    assert stats(n=0, h=None, lse=None, g=None, k=None) == 0
    assert stats(a=3, b=3, g=None, k=None) == 0


def test_workspace_bytes():
    assert B.gbdt_leaf_product_grad_workspace_bytes(-1, 8, 8) == 0
    assert B.gbdt_leaf_product_grad_workspace_bytes(8, 0, 8) == 0
    assert B.gbdt_leaf_product_grad_workspace_bytes(400, 64, 64) < B.gbdt_leaf_product_grad_workspace_bytes(40_000, 64, 64)
    # bounded by the compute units, not by the sizes
    assert B.gbdt_leaf_product_grad_workspace_bytes(400_000, 2000, 256) < 512 << 20
    assert B.gbdt_softmax_workspace_bytes(8, 0, 8) == 0
    # the scores of 8,192 rows over 65,536 classes would take 2 GiB in 32 bits
    assert 0 < B.gbdt_softmax_workspace_bytes(8192, 65536, 1024, torch.bfloat16) < 1 << 30


def test_the_oracle_agrees_with_automatic_differentiation():
    """The oracle's own formulas against torch's gradients of a loss written another way, on the CPU in 64 bits."""
    g = torch.Generator().manual_seed(0)
    n, v, dim, leaves, d_in = 40, 23, 6, 3, 5
    x = torch.randn(n, d_in, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(leaves, dim, d_in, generator=g, dtype=torch.float64, requires_grad=True)
    b = torch.randn(leaves, dim, generator=g, dtype=torch.float64, requires_grad=True)
    c = torch.randn(v, dim, generator=g, dtype=torch.float64, requires_grad=True)
    y = torch.randint(-1, v + 1, (n,), generator=g, dtype=torch.int32)
    rw = torch.rand(n, generator=g, dtype=torch.float64)
    order = torch.randperm(n, generator=g).to(torch.int32)
    offs = [0, 13, 13, 40]
    leaf_id = torch.empty(n, dtype=torch.long)
    for l in range(leaves):
        leaf_id[order[offs[l]:offs[l + 1]].long()] = l
    h = (w[leaf_id] * x[:, None, :]).sum(2) + b[leaf_id]
    use = (y >= 0) & (y < v)
    logp = torch.log_softmax((h[:, None, :] * c[None]).sum(2), 1)
    each = torch.where(use, -logp[torch.arange(n), torch.where(use, y, torch.zeros_like(y)).long()], torch.zeros(n, dtype=torch.float64))
    h.retain_grad()
    (0.3 * rw * each).sum().backward()
    got_h, _ = ref.leaf_product(x.detach(), w.detach(), b.detach(), offs, order, torch.zeros(n, dim, dtype=torch.float64))
    assert torch.allclose(got_h, h.detach(), atol=1e-12)
    got_loss, lse = ref.softmax_loss(got_h, c.detach(), y)
    assert torch.allclose(got_loss, each.detach(), atol=1e-12)
    (dh, dc), _ = ref.softmax_grad(got_h, c.detach(), y, lse, rw, 0.3)
    assert torch.allclose(dh, h.grad, atol=1e-12) and torch.allclose(dc, c.grad, atol=1e-12)
    (dx, dw, db), _ = ref.leaf_product_grad(dh, x.detach(), w.detach(), offs, order, torch.zeros_like(x.detach()))
    assert torch.allclose(dx, x.grad, atol=1e-12) and torch.allclose(dw, w.grad, atol=1e-12) and torch.allclose(db, b.grad, atol=1e-12)
    grad, hess = ref.softmax_stats(got_h, c.detach(), y, lse, 4, 9)
    p = torch.exp(logp.detach()).t()[4:9] * use
    assert torch.allclose(hess, p * (1 - p), atol=1e-12)
    assert torch.allclose(grad, p - (y[None, :] == torch.arange(4, 9)[:, None]).double(), atol=1e-12)
