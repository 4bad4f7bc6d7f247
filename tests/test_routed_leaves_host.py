"""What the calls of routed rows and of 8-bit codes refuse, before any GPU work (addresses here are never followed), and the oracle
against gradients by differences and by automatic differentiation."""
import math

import pytest
import torch

from oracle import routed_leaves as ref
from paper_1706_08359_amd import binding as B

P, EINVAL, EUNSUPPORTED = 4096, -1, -2


def route(l=P, ld=8, bias=P, n=5, leaves=8, dtype=0, score=0, groups=1, kept=1, best=1, k=2, renorm=1, scale=1.0, out=P, gates=P):
    return B.load().gbdt_route(l, ld, bias, n, leaves, dtype, score, groups, kept, best, k, renorm, scale, out, gates, None)


def route_grad(l=P, ld=8, e=P, dg=P, n=5, leaves=8, dtype=0, score=0, k=2, renorm=1, scale=1.0, out=P, ld_out=8):
    return B.load().gbdt_route_grad(l, ld, e, dg, n, leaves, dtype, score, k, renorm, scale, out, ld_out, None)


def mixture(x=P, ld_x=8, w=P, b=P, e=P, g=P, n=5, k=2, leaves=3, d_in=8, d_out=4, dtype=0, y=P, ld_y=4):
    return B.load().gbdt_mixture_product(x, ld_x, w, b, e, g, n, k, leaves, d_in, d_out, dtype, y, ld_y, None)


def mixture_grad(dy=P, ld_dy=4, x=P, ld_x=8, w=P, b=P, e=P, g=P, n=5, k=2, leaves=3, d_in=8, d_out=4, dtype=0, dx=P, ld_dx=8, dw=P,
                 db=P, dg=P):
    return B.load().gbdt_mixture_product_grad(dy, ld_dy, x, ld_x, w, b, e, g, n, k, leaves, d_in, d_out, dtype, dx, ld_dx, dw, db, dg,
                                              None)


def quantize(x=P, ld=20, n=5, cols=20, dtype=0, codes=P, ld_codes=32, scales=P):
    return B.load().gbdt_rows_quantize(x, ld, n, cols, dtype, codes, ld_codes, scales, None)


def leaf_codes(c=P, ld=32, s=P, w=P, ws=P, b=P, idx=P, offs=P, pos=5, leaves=3, n=5, d_in=20, d_out=4, dtype=0, y=P, ld_y=4):
    return B.load().gbdt_leaf_product_codes(c, ld, s, w, ws, b, idx, offs, pos, leaves, n, d_in, d_out, dtype, y, ld_y, None)


def mixture_codes(c=P, ld=32, s=P, w=P, ws=P, b=P, e=P, g=P, n=5, k=2, leaves=3, d_in=20, d_out=4, dtype=0, y=P, ld_y=4):
    return B.load().gbdt_mixture_product_codes(c, ld, s, w, ws, b, e, g, n, k, leaves, d_in, d_out, dtype, y, ld_y, None)


REFUSED = [
    (route, [dict(l=None), dict(l=P + 2), dict(l=P + 1, dtype=1), dict(ld=7), dict(n=-1), dict(leaves=0), dict(dtype=2), dict(score=2),
             dict(score=-1), dict(groups=0), dict(groups=3), dict(kept=0), dict(groups=2, kept=3), dict(best=0), dict(best=3), dict(k=0),
             dict(k=9), dict(groups=4, kept=1, k=3), dict(scale=math.nan), dict(scale=math.inf), dict(out=None), dict(gates=None),
             dict(bias=P + 2), dict(out=P + 1), dict(gates=P + 2)]),
    (route_grad, [dict(l=None), dict(e=None), dict(dg=None), dict(out=None), dict(ld=7), dict(ld_out=7), dict(n=-1), dict(leaves=0),
                  dict(dtype=3), dict(score=2), dict(k=0), dict(k=9), dict(scale=math.inf), dict(out=P + 2), dict(e=P + 1), dict(dg=P + 2)]),
    (mixture, [dict(x=None), dict(w=None), dict(e=None), dict(g=None), dict(y=None), dict(ld_x=7), dict(ld_y=3), dict(n=-1), dict(k=0),
               dict(leaves=0), dict(d_in=0), dict(d_out=0), dict(dtype=2), dict(x=P + 2), dict(w=P + 1, dtype=1), dict(b=P + 2),
               dict(y=P + 2), dict(e=P + 2), dict(g=P + 1)]),
    (mixture_grad, [dict(dy=None), dict(x=None), dict(w=None), dict(e=None), dict(g=None), dict(ld_dy=3), dict(ld_x=7), dict(ld_dx=7),
                    dict(n=-1), dict(k=0), dict(leaves=0), dict(d_in=0), dict(dtype=2), dict(dx=P + 2), dict(dw=P + 1), dict(db=P + 2),
                    dict(dg=P + 2), dict(dy=P + 1, dtype=1), dict(dx=None, dw=None, db=None, x=None)]),
    (quantize, [dict(x=None), dict(codes=None), dict(scales=None), dict(ld=19), dict(ld_codes=20), dict(ld_codes=16), dict(ld_codes=40),
                dict(codes=P + 8), dict(x=P + 2), dict(n=-1), dict(cols=0), dict(dtype=2), dict(scales=P + 2)]),
    (leaf_codes, [dict(c=None), dict(s=None), dict(w=None), dict(ws=None), dict(offs=None), dict(y=None), dict(ld=20), dict(ld=40),
               dict(c=P + 8), dict(w=P + 8), dict(ld_y=3), dict(pos=-1), dict(leaves=0), dict(n=-1), dict(d_in=0), dict(d_out=0),
               dict(dtype=2), dict(idx=None, pos=6), dict(b=P + 2), dict(y=P + 2), dict(offs=P + 4), dict(idx=P + 2)]),
    (mixture_codes, [dict(c=None), dict(s=None), dict(w=None), dict(ws=None), dict(e=None), dict(g=None), dict(y=None), dict(ld=16),
                  dict(ld=40), dict(k=0), dict(c=P + 4), dict(ld_y=3), dict(dtype=5)]),
]


@pytest.mark.parametrize("call,bad", [(c, b) for c, many in REFUSED for b in many], ids=lambda v: getattr(v, "__name__", str(v)))
def test_refuses(call, bad):
    assert call(**bad) == EINVAL


@pytest.mark.parametrize("call,big", [
    (route, dict(n=1 << 30)), (route, dict(leaves=1025, ld=1025)), (route, dict(leaves=64, ld=64, k=33)),
    (route, dict(leaves=130, ld=130, groups=65)), (route, dict(ld=1 << 28)), (route_grad, dict(ld_out=1 << 28)),
    (route_grad, dict(leaves=1025, ld=1025, ld_out=1025)), (mixture, dict(n=1 << 30)), (mixture, dict(k=65)),
    (mixture, dict(n=1 << 25, k=32)), (mixture, dict(leaves=16385)), (mixture, dict(d_in=1 << 24, ld_x=1 << 24)),
    (mixture, dict(d_out=1 << 24, ld_y=1 << 24)), (mixture_grad, dict(leaves=16385)), (mixture_grad, dict(ld_dx=1 << 28)),
    (quantize, dict(n=1 << 30)), (quantize, dict(ld=1 << 28)), (leaf_codes, dict(d_in=131073, ld=131088)),
    (mixture_codes, dict(d_in=131073, ld=131088)), (mixture_codes, dict(k=65)), (leaf_codes, dict(leaves=1 << 24))],
    ids=lambda v: getattr(v, "__name__", str(v)))
def test_limits(call, big):
    assert call(**big) == EUNSUPPORTED


def test_nothing_to_do():
    assert route(n=0, l=None, out=None, gates=None) == 0
    assert route_grad(n=0, l=None, e=None, dg=None, out=None) == 0
    assert mixture(n=0, x=None, e=None, g=None, y=None) == 0
    assert mixture_grad(n=0, dy=None, x=None, e=None, g=None, dw=None, db=None) == 0
    assert mixture_grad(dx=None, dw=None, db=None, dg=None) == 0
    assert quantize(n=0, x=None, codes=None, scales=None) == 0
    assert leaf_codes(pos=0, c=None, s=None, y=None) == 0
    assert mixture_codes(n=0, c=None, s=None, y=None, e=None, g=None) == 0


def test_workspace_bytes():
    size = B.gbdt_mixture_workspace_bytes
    assert size(-1, 2, 3, 8, 8) == 0 and size(8, 65, 3, 8, 8) == 0 and size(8, 2, 0, 8, 8) == 0 and size(8, 2, 16385, 8, 8) == 0
    assert 0 < size(100, 2, 64, 64, 64) < size(10_000, 2, 64, 64, 64)
    # slots of 400,000 rows x 8 leaves x 2,000 values would take 25 GB
    assert size(400_000, 8, 255, 2000, 128) < 2 << 30
    # and so would weighted gradients of 2,000 outputs take 13 GB: 128 at a time
    assert size(400_000, 8, 255, 128, 2000, torch.bfloat16) < 2 << 30
    # never less for more rows
    many = [size(n, 3, 300, 40, 24) for n in range(1, 400_000, 7001)]
    assert many == sorted(many)


CASES = [dict(score=s, renormalise=r) for s in ("softmax", "sigmoid") for r in (True, False)]


@pytest.mark.parametrize("how", CASES, ids=str)
def test_the_oracles_gradient_of_logits(how):
    """Against central differences of its own weights with the choice held, whose error is h^2 of a third derivative."""
    g = torch.Generator().manual_seed(3)
    logits = torch.randn(6, 9, generator=g, dtype=torch.float64)
    leaves, gates = ref.route(logits, 3, scale=1.7, **how)
    dg = torch.randn(6, 3, generator=g)
    got, _ = ref.route_grad(logits, leaves, dg, scale=1.7, **how)
    want, h = torch.zeros_like(got), 1e-4
    for e in range(9):
        step = torch.zeros(9, dtype=torch.float64)
        step[e] = h
        up, down = (ref.weights(logits + v, leaves, how["score"], how["renormalise"], 1.7) for v in (step, -step))
        want[:, e] = ((up - down) * dg.double()).sum(1) / (2 * h)
    assert torch.allclose(got, want, atol=1e-7)


def test_the_oracles_choice():
    inf = math.inf
    logits = torch.tensor([[1.0, 3.0, 3.0, -inf, 2.0, math.nan], [-inf] * 6, [0.0] * 6, [5.0, -inf, -inf, -inf, -inf, math.nan]])
    leaves, gates = ref.route(logits, 3)
    assert leaves.tolist() == [[1, 2, 4], [-1, -1, -1], [0, 1, 2], [0, -1, -1]]
    assert torch.allclose(gates[2], torch.full((3,), 1 / 3, dtype=torch.float64)) and gates[3].tolist() == [1.0, 0.0, 0.0]
    assert gates[1].tolist() == [0.0, 0.0, 0.0]
    # a bias moves the choice, not the weights
    leaves, gates = ref.route(logits[2:3], 2, choice_bias=torch.tensor([0.0, 0, 0, 1, 0, 2]), score="sigmoid", renormalise=False)
    assert leaves.tolist() == [[5, 3]] and gates.tolist() == [[0.5, 0.5]]
    # groups: by their two largest together, (3 + 0), (2 + 1.5), (2.9 + 0.2)
    l = torch.tensor([[3.0, 0.0, 2.0, 1.5, 2.9, 0.2]])
    bias = torch.zeros(6)
    assert ref.route(l, 2, n_groups=3, groups_kept=1)[0].tolist() == [[0, 1]]
    s = torch.sigmoid(l.double())[0]
    pair = [float(s[0] + s[1]), float(s[2] + s[3]), float(s[4] + s[5])]
    best = max(range(3), key=lambda q: pair[q])
    assert ref.route(l, 2, choice_bias=bias, score="sigmoid", n_groups=3, groups_kept=1, group_best=2)[0].tolist() == [[2 * best, 2 * best + 1]]


def test_the_oracles_mixture_against_automatic_differentiation():
    g = torch.Generator().manual_seed(0)
    n, k, leaves, d_in, d_out = 11, 3, 5, 7, 4
    f64 = dict(generator=g, dtype=torch.float64)
    x = torch.randn(n, d_in, **f64, requires_grad=True)
    w = torch.randn(leaves, d_out, d_in, **f64, requires_grad=True)
    b = torch.randn(leaves, d_out, **f64, requires_grad=True)
    gates = torch.rand(n, k, **f64, requires_grad=True)
    e = torch.randint(-1, leaves + 1, (n, k), generator=g, dtype=torch.int32)
    e[0] = -1
    e[1] = 2
    use = (e >= 0) & (e < leaves)
    at = torch.where(use, e, 0).long()
    y = ((w[at] * x[:, None, None, :]).sum(3) + b[at]) * torch.where(use, gates, 0.0)[:, :, None]
    y = y.sum(1)
    dy = torch.randn(n, d_out, **f64)
    (y * dy).sum().backward()
    data = [v.detach() for v in (x, w, b)]
    got, _ = ref.mixture(*data, e, gates.detach())
    assert torch.allclose(got, y.detach(), atol=1e-12) and got[0].abs().sum() == 0
    (dx, dw, db, dg), _ = ref.mixture_grad(dy, *data, e, gates.detach())
    for a, v in ((dx, x), (dw, w), (db, b), (dg, gates)):
        assert torch.allclose(a, v.grad, atol=1e-12)


def test_the_oracles_codes():
    x = torch.tensor([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5], [0.0] * 6, [math.inf, 1, 2, 3, 4, 5], [1e-40] * 6, [math.nan, 0, 0, 0, 0, 0]])
    codes, scales = ref.quantize(x)
    # (127 / 127 is 1 with the 32-bit 1 / 127 too)
    assert codes[0].tolist() == [127, -127, 0, 2, 2, 0] and scales[0] == 1.0
    assert codes[1:].abs().sum() == 0 and scales[1] == 0 and scales[3] == 0
    assert torch.isnan(scales[2]) and torch.isnan(scales[4])
