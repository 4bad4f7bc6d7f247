"""The calls of routed rows together, as routed_leaves uses them."""
import pytest
import torch

from oracle import linear_leaves as one_leaf
from oracle import routed_leaves as ref

pytestmark = pytest.mark.gpu


def small(dtype, score, seed=0, **kw):
    from paper_1706_08359_amd import linear_leaves as L
    from paper_1706_08359_amd import routed_leaves as R
    x, _, _, labels, n_classes = L.synthetic(n_rows=1200, n_classes=40, seed=seed, dtype=dtype)
    labels[::9] = -1
    model = R.Mixture(28, 12, 3, n_classes, dim=8, score=score, dtype=dtype, seed=seed, **kw)
    model.choice_bias += 0.01 * torch.randn(12, generator=torch.Generator().manual_seed(7)).cuda()
    return x, labels, model


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 0.03)])
def test_the_gradients_of_a_step_are_the_formulas(dtype, tol, score):
    """Against the 64-bit definitions chained together, from the same choice of leaves.  f32: sums of at most 3,600 terms and a handful
    of roundings.  bf16: logits, embeddings, dh, dlogits and gates * dh are rounded between the calls, 2^-8 each."""
    x, labels, model = small(dtype, score)
    _, grads, taken = model.gradients(x, labels)
    assert int(taken.sum()) == 1200 * 3
    router, weight, bias, classes = model._copies()
    logits, leaves, _ = model.route(x, router)
    assert torch.equal(leaves, ref.route(logits, 3, choice_bias=model.choice_bias, score=score)[0])
    offs = [0, 1200]
    logits64, _ = one_leaf.leaf_product(x, router, None, offs, None, torch.zeros(1200, 12, device="cuda"))
    gates64 = ref.weights(logits64, leaves, score, True, 1.0)
    h64, _ = ref.mixture(x, weight, bias, leaves, gates64)
    _, lse64 = one_leaf.softmax_loss(h64, classes, labels)
    counted = int((labels >= 0).sum())
    (dh64, dc64), _ = one_leaf.softmax_grad(h64, classes, labels, lse64, None, 1 / counted)
    (_, dw64, db64, dg64), _ = ref.mixture_grad(dh64, x, weight, bias, leaves, gates64)
    dl64, _ = ref.route_grad(logits64, leaves, dg64, score=score)
    (_, dr64, _), _ = one_leaf.leaf_product_grad(dl64, x, router, offs, None, torch.zeros(1200, 28, device="cuda"))
    for name, got, want in zip(("router", "weight", "bias", "classes"), grads, (dr64, dw64, db64, dc64)):
        assert float((got.double() - want).norm()) <= tol * float(want.norm()), name


def test_gradients_against_differences_of_the_loss():
    """Central differences of the 64-bit loss, leaves held, along one direction of all parameters: h^2 of a third derivative and the
    f32 gradients' roundings."""
    x, labels, model = small(torch.float32, "sigmoid", seed=3)
    _, grads, _ = model.gradients(x, labels)
    params = model._copies()
    leaves = model.route(x)[1]
    g = torch.Generator().manual_seed(4)
    steps = [torch.randn(p.shape, generator=g).cuda().double() for p in params]

    def loss(t):
        router, weight, bias, classes = (p.double() + t * s for p, s in zip(params, steps))
        logits, _ = one_leaf.leaf_product(x, router, None, [0, 1200], None, torch.zeros(1200, 12, device="cuda"))
        h, _ = ref.mixture(x, weight, bias, leaves, ref.weights(logits, leaves, "sigmoid", True, 1.0))
        each, _ = one_leaf.softmax_loss(h, classes, labels)
        return float(each.sum()) / int((labels >= 0).sum())
    h = 1e-4
    diff = (loss(h) - loss(-h)) / (2 * h)
    want = sum(float((d.double() * s).sum()) for d, s in zip(grads, steps))
    size = sum(float((d.double() * s).abs().sum()) for d, s in zip(grads, steps))
    assert abs(diff - want) <= 1e-5 * size + 1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_run_and_answers_agree(dtype):
    x, labels, model = small(dtype, "sigmoid", n_groups=4, groups_kept=2)
    for _ in range(5):
        loss = model.step(x, labels, rate=2.0)
        assert loss == loss
    y = model.answer(x)
    few = model.answer(x[:1])
    assert float((few.double() - y[:1].double()).norm()) <= 0.02 * float(y[:1].double().norm())
    codes = model.quantized()
    _, leaves, gates = model.route(x)
    q = codes.answer(x, leaves, gates)
    want, _ = ref.mixture(*decoded(codes, x), leaves, gates)
    assert float((q.double() - want).norm()) <= 1e-6 * float(want.norm())


def decoded(codes, x):
    c, s = ref.quantize(x)
    return c.double() * s.double()[:, None], codes.weight[:, :, :x.shape[1]].double() * codes.scales.double()[:, :, None], codes.bias


@pytest.mark.parametrize("trees", [3, 70])
def test_a_forest_is_a_mixture(trees):
    """The trees of a model answered in one call are what they are one after another, up to the order of f32 sums; and in 8 bits, what the
    codes stand for."""
    from paper_1706_08359_amd import binding as B
    from paper_1706_08359_amd import linear_leaves as L
    from paper_1706_08359_amd import routed_leaves as R
    x, bins, n_bins, labels, n_classes = L.synthetic(n_rows=900, n_classes=30, seed=6)
    model = L.Model(x, bins, n_bins, labels, n_classes, dim=8)
    for _ in range(trees):
        model.add_tree(max_leaves=5, steps=1, rate=2.0)
    leaves, gates = R.forest_leaves(model, bins)
    weight, bias = R.forest(model)
    assert leaves.shape == (900, trees)
    if trees <= 64:
        y = B.gbdt_mixture_product(x, weight, leaves, gates, bias=bias)
        want, mag = ref.mixture(x, weight, bias, leaves, gates)
        assert bool(((y.double() - want).abs() <= (28 + trees + 3) * 2.0 ** -24 * mag).all())
        assert bool(((y.double() - model.embed_rows(x, bins).double()).abs() <= 2 * (28 + trees + 3) * 2.0 ** -24 * mag).all())
    codes = R.Codes(weight, bias)
    q = codes.answer(x, leaves, gates)
    want, mag = ref.mixture(*decoded(codes, x), leaves, gates)
    assert bool(((q.double() - want).abs() <= (trees + 8) * 2.0 ** -24 * mag).all())


def test_the_example_runs(capsys):
    from paper_1706_08359_amd import routed_leaves as R
    R.main(steps=3)
    out = capsys.readouterr().out
    assert "step 2" in out and "one row" in out
