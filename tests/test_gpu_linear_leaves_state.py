"""What a bf16 model adds to tree after tree is kept in 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def small(**kw):
    from paper_1706_08359_amd import linear_leaves as L
    x, bins, n_bins, labels, n_classes = L.synthetic(n_rows=1500, n_classes=40, seed=5, dtype=torch.bfloat16)
    return x, bins, L.Model(x, bins, n_bins, labels, n_classes, dim=8, **kw)


def test_embeddings_of_many_trees():
    """The rounding of 48 trees' sum is that of one bf16 value, 2^-8 of itself at most, and what 48 f32 sums add."""
    x, bins, model = small()
    for _ in range(48):
        model.add_tree(max_leaves=4, steps=1, rate=2.0)
    trees, total, mag = model.trees, 0.0, 0.0
    assert torch.equal(model.embed_rows(x, bins), model.embed)
    for tree in trees:
        model.trees = [tree]
        one = model.embed_rows(x, bins).double()
        total, mag = total + one, mag + one.abs()
    model.trees = trees
    assert model.embed.dtype == torch.bfloat16
    err = (model.embed.double() - total).abs()
    assert bool((err <= 2.0 ** -8 * total.abs() + 50 * 2.0 ** -24 * mag).all()), float(err.max())


def test_steps_of_the_classes_add_up(monkeypatch):
    """20 trees, each with a step of 0.001 from 1, below half of what bf16 keeps there."""
    from paper_1706_08359_amd import linear_leaves as L
    x, bins, model = small()
    model.classes = torch.ones_like(model.classes)
    real = L.B.gbdt_softmax_grad
    monkeypatch.setattr(L.B, "gbdt_softmax_grad", lambda h, c, *a, **k: (real(h, c, *a, **k)[0], torch.full_like(c, 0.125)))
    for _ in range(20):
        model.add_tree(max_leaves=3, steps=1, rate=0.008)
    assert model.classes.dtype == torch.bfloat16
    assert float((model.classes.double() - 0.98).abs().max()) <= 2.0 ** -9 + 1e-5


def test_what_is_set_is_what_is_read():
    x, bins, model = small()
    embed, classes = torch.randn_like(model.embed), torch.randn_like(model.classes)
    model.embed, model.classes = embed, classes
    assert torch.equal(model.embed, embed) and torch.equal(model.classes, classes)
    loss, lse = model.loss()
    want = torch.logsumexp(embed.double() @ classes.double().t().contiguous(), 1)
    assert float((lse.double() - want).abs().max()) < 1e-4 * float(want.abs().max())
