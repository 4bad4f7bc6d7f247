"""Rows that several linear leaves answer: the calls of the binding as a trainer and a server use them together.

`Mixture` learns which leaves answer a row instead of growing a tree for it.  One step
  1. scores the leaves (gbdt_leaf_product with the router's matrix as the only leaf) and chooses k of them (gbdt_route),
  2. answers with their weighted products (gbdt_mixture_product), an embedding that a matrix of classes turns into scores,
  3. takes the loss and all gradients (gbdt_softmax_loss, gbdt_softmax_grad, gbdt_mixture_product_grad, gbdt_route_grad,
     gbdt_leaf_product_grad),
  4. moves the choice bias of leaves that are taken too often or too seldom, which no gradient does.
`Mixture.quantized` and `forest` hold a trained mixture, or the trees of linear_leaves.Model, in 8 bits: `Codes.answer` quantizes rows
and answers them (gbdt_rows_quantize, gbdt_mixture_product_codes).

    python -m paper_1706_08359_amd.routed_leaves        # a small synthetic run; prints the loss now and then
"""
from __future__ import annotations

import torch

from . import binding as B
from . import linear_leaves as L

MAX_LEAVES_A_ROW, MAX_LEAVES = 64, 16384   # of one call; a forest of more trees, or of more leaves in all, takes several


class Codes:
    """Matrices of linear leaves as 8-bit codes: weight [n_leaves, d_out, d_in], bias [n_leaves, d_out]."""

    def __init__(self, weight, bias):
        n_leaves, d_out, d_in = weight.shape
        codes, scales = B.gbdt_rows_quantize(weight.reshape(n_leaves * d_out, d_in))
        self.weight, self.scales = codes.view(n_leaves, d_out, -1), scales.view(n_leaves, d_out)
        self.bias = bias.float().contiguous()

    def answer(self, x, leaves, gates, dtype=torch.float32):
        """sum_j gates[d, j] (W_l x[d] + b_l), rows quantized in the call."""
        return self.answer_codes(*B.gbdt_rows_quantize(x), leaves, gates, dtype)

    def answer_codes(self, codes, scales, leaves, gates, dtype=torch.float32):
        """The same of rows that are held as codes."""
        y, n_leaves = None, self.weight.shape[0]
        for first in range(0, max(1, n_leaves), MAX_LEAVES):
            # (the others are outside this part's leaves, and passed over)
            matrices = [t[first:first + MAX_LEAVES] for t in (self.weight, self.scales, self.bias)]
            here = leaves - first if first else leaves
            for a in range(0, max(1, leaves.shape[1]), MAX_LEAVES_A_ROW):
                part = [t[:, a:a + MAX_LEAVES_A_ROW].contiguous() for t in (here, gates)]
                z = B.gbdt_mixture_product_codes(codes, scales, *matrices[:2], *part, bias=matrices[2], dtype=torch.float32)
                y = z if y is None else y + z
        return y.to(dtype)


def forest_leaves(model, bins):
    """(leaves int32 [n_rows, trees], gates) of rows in the trees of a linear_leaves.Model, leaves numbered through all trees."""
    columns, first = [], 0
    for nodes, leaves, _, _ in model.trees:
        row_idx, offsets = L.route(nodes, bins, leaves)
        column = torch.empty(bins.shape[0], dtype=torch.int32, device=bins.device)
        numbers = torch.arange(first, first + len(leaves), dtype=torch.int32, device=bins.device)
        column[row_idx.long()] = torch.repeat_interleave(numbers, offsets[1:] - offsets[:-1])
        columns.append(column)
        first += len(leaves)
    leaves = torch.stack(columns, 1).contiguous()
    return leaves, torch.ones(leaves.shape, device=leaves.device)


def forest(model):
    """(weight, bias) of all leaves of a linear_leaves.Model's trees, as gbdt_mixture_product and Codes take them."""
    return torch.cat([w for _, _, w, _ in model.trees]).contiguous(), torch.cat([b for _, _, _, b in model.trees]).contiguous()


class Mixture:
    """x: [n_rows, n_features] float32 or bfloat16; labels: int32 (outside [0, n_classes): the row is left out).  What steps are
    added to is kept in 32 bits; the products read copies of x's type."""

    def __init__(self, n_features, n_leaves, k, n_classes, dim, score="sigmoid", n_groups=1, groups_kept=1, dtype=torch.float32,
                 device="cuda", seed=0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.k, self.dtype, self.score = k, dtype, score
        self.groups = dict(n_groups=n_groups, groups_kept=groups_kept)
        made = dict(generator=gen, device=device)
        self.router = torch.randn(1, n_leaves, n_features, **made) * n_features ** -0.5
        self.weight = torch.randn(n_leaves, dim, n_features, **made) * n_features ** -0.5
        self.bias = torch.zeros(n_leaves, dim, device=device)
        self.classes = torch.randn(n_classes, dim, **made) * dim ** -0.5
        self.choice_bias = torch.zeros(n_leaves, device=device)

    def _copies(self):
        return [t.to(self.dtype) for t in (self.router, self.weight, self.bias, self.classes)]

    def route(self, x, router=None):
        """(logits, leaves, gates) of rows."""
        router = self.router.to(self.dtype) if router is None else router
        one_leaf = torch.tensor([0, x.shape[0]], dtype=torch.int64, device=x.device)
        logits = B.gbdt_leaf_product(x, router, one_leaf)
        leaves, gates = B.gbdt_route(logits, self.k, choice_bias=self.choice_bias, score=self.score, **self.groups)
        return logits, leaves, gates

    def gradients(self, x, labels):
        """(mean loss, gradients of (router, weight, bias, classes) by it, rows that took each leaf)."""
        router, weight, bias, classes = self._copies()
        n_classes, n_leaves = classes.shape[0], weight.shape[0]
        counted = max(1, int(((labels >= 0) & (labels < n_classes)).sum()))
        logits, leaves, gates = self.route(x, router)
        h = B.gbdt_mixture_product(x, weight, leaves, gates, bias=bias)
        loss, lse = B.gbdt_softmax_loss(h, classes, labels)
        dh, dclasses = B.gbdt_softmax_grad(h, classes, labels, lse, scale=1.0 / counted)
        _, dweight, dbias, dgates = B.gbdt_mixture_product_grad(dh, x, weight, leaves, gates, bias=bias,
                                                                want=("weight", "bias", "gates"))
        dlogits = B.gbdt_route_grad(logits, leaves, dgates, score=self.score)
        one_leaf = torch.tensor([0, x.shape[0]], dtype=torch.int64, device=x.device)
        _, drouter, _ = B.gbdt_leaf_product_grad(dlogits, x, router, one_leaf, want=("weight",))
        taken = torch.bincount(leaves[leaves >= 0], minlength=n_leaves)
        return float(loss.double().sum()) / counted, (drouter, dweight, dbias, dclasses), taken

    def step(self, x, labels, rate=1.0, balance=1e-3):
        """One gradient step; returns the mean loss before it."""
        loss, grads, taken = self.gradients(x, labels)
        for t, d in zip((self.router, self.weight, self.bias, self.classes), grads):
            t -= rate * d.float()
        mean = taken.double().mean()
        self.choice_bias += balance * torch.sign(mean - taken.double()).float()
        return loss

    def answer(self, x):
        """Embeddings of rows; one row is answered as well as many."""
        _, weight, bias, _ = self._copies()
        _, leaves, gates = self.route(x)
        return B.gbdt_mixture_product(x, weight, leaves, gates, bias=bias)

    def quantized(self):
        return Codes(self.weight.to(self.dtype), self.bias)


def main(steps=60):
    x, _, _, labels, n_classes = L.synthetic()
    model = Mixture(x.shape[1], 16, 2, n_classes, dim=16)
    for s in range(steps):
        loss = model.step(x, labels, rate=8.0)
        if s % 10 == 0 or s == steps - 1:
            print("step %d: loss %.4f" % (s, loss), flush=True)
    codes = model.quantized()
    _, leaves, gates = model.route(x[:1])
    print("one row: leaves %s, 8-bit answers off by %.4f of their size" % (
        leaves[0].tolist(), float((codes.answer(x[:1], leaves, gates) - model.answer(x[:1])).norm() / model.answer(x[:1]).norm())), flush=True)


if __name__ == "__main__":
    main()
