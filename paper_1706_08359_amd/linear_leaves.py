"""Trees with linear leaves for many classes: the calls of the binding as a trainer uses them together.

A row's answer is an embedding, the sum over trees of `weight[leaf] x + bias[leaf]`; a matrix of classes turns it into the
scores of a softmax.  One round of `Model.add_tree`
  1. takes the loss of the present embeddings (gbdt_softmax_loss) and the gradient and hessian columns of the class with
     the largest sum of squared gradients among a few (gbdt_softmax_stats),
  2. grows a tree on them (gbdt_grow_tree), whose row order lists the rows of its leaves,
  3. trains the leaves' matrices and the classes by gradient steps (gbdt_leaf_product, gbdt_softmax_loss, gbdt_softmax_grad,
     gbdt_leaf_product_grad).
Nothing of the size of rows x classes is ever held.

    python -m paper_1706_08359_amd.linear_leaves        # a small synthetic run; prints the loss after every tree
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


def leaf_lists(nodes: np.ndarray, device):
    """(leaf ids in the order of their rows, leaf_offsets) of a grown tree: gbdt_leaf_product's grouping of row_order."""
    leaves = np.flatnonzero(nodes["left"] < 0)
    leaves = leaves[np.argsort(nodes["row_begin"][leaves], kind="stable")]
    offsets = np.zeros(len(leaves) + 1, dtype=np.int64)
    offsets[:-1] = nodes["row_begin"][leaves]
    offsets[-1] = nodes["row_begin"][leaves[-1]] + nodes["count"][leaves[-1]]
    return leaves, torch.from_numpy(offsets).to(device)


def route(nodes: np.ndarray, bins: torch.Tensor, leaves: np.ndarray):
    """(row_idx, leaf_offsets) of other rows, by their bins: what gbdt_leaf_product takes, grouped as `leaves` is ordered."""
    table = {k: torch.from_numpy(nodes[k].astype(np.int64)).to(bins.device) for k in ("left", "right", "feature", "bin")}
    node = torch.zeros(bins.shape[0], dtype=torch.int64, device=bins.device)
    while True:
        open_ = table["left"][node] >= 0
        if not bool(open_.any()):
            break
        f = table["feature"][node].clamp(min=0)
        left = bins.gather(1, f[:, None])[:, 0].long() <= table["bin"][node]
        node = torch.where(open_, torch.where(left, table["left"][node], table["right"][node]), node)
    rank = torch.full((len(nodes),), -1, dtype=torch.int64, device=bins.device)
    rank[torch.from_numpy(leaves).to(bins.device)] = torch.arange(len(leaves), device=bins.device)
    leaf = rank[node]
    offsets = torch.zeros(len(leaves) + 1, dtype=torch.int64, device=bins.device)
    offsets[1:] = torch.cumsum(torch.bincount(leaf, minlength=len(leaves)), 0)
    return torch.sort(leaf, stable=True)[1].to(torch.int32), offsets


class Model:
    """x: [n_rows, n_features] float32 or bfloat16, the values the leaves are linear in; bins: uint8 of the same rows, what
    the trees split on; labels: int32 (outside [0, n_classes): the row is left out of the training).
    What is added to tree after tree, the rows' embeddings and the classes, is kept in 32 bits; `embed` and `classes` are
    rounded to x's type, as the products take them."""

    def __init__(self, x, bins, n_bins, labels, n_classes, dim, seed=0):
        gen = torch.Generator(device=x.device)
        gen.manual_seed(seed)
        self.x, self.bins, self.n_bins, self.labels = x, bins, n_bins, labels
        self.packed = B.gbdt_bins_pack(bins, n_bins)
        self.n_rows, self.n_classes = x.shape[0], n_classes
        self._classes = (torch.randn(n_classes, dim, generator=gen, device=x.device) * dim ** -0.5).to(x.dtype).float()
        self._embed = torch.zeros(self.n_rows, dim, device=x.device)
        self.counted = int(((labels >= 0) & (labels < n_classes)).sum())
        self.trees = []

    @property
    def classes(self):
        return self._classes.to(self.x.dtype)

    @classes.setter
    def classes(self, value):
        self._classes = value.float()

    @property
    def embed(self):
        return self._embed.to(self.x.dtype)

    @embed.setter
    def embed(self, value):
        self._embed = value.float()

    def loss(self):
        """(mean loss over the rows that count, lse)."""
        loss, lse = B.gbdt_softmax_loss(self.embed, self.classes, self.labels)
        return float(loss.double().sum()) / max(self.counted, 1), lse

    def add_tree(self, max_leaves=31, steps=10, rate=1.0, lam=1.0, min_child_hess=1e-3, candidates=16):
        """Grows a tree, trains its leaves and the classes; returns the mean loss after the last step's gradient."""
        embed, classes = self.embed, self.classes
        _, lse = B.gbdt_softmax_loss(embed, classes, self.labels)
        begin = (len(self.trees) * candidates) % max(1, self.n_classes - candidates + 1)
        grad, hess = B.gbdt_softmax_stats(embed, classes, self.labels, lse, begin,
                                          min(self.n_classes, begin + candidates))
        k = int((grad.double() ** 2).sum(1).argmax())
        nodes, row_idx, _ = B.gbdt_grow_tree(self.packed, self.n_rows, self.bins.shape[1], self.n_bins, grad[k], hess[k],
                                             max_leaves, lam, min_child_hess)
        leaves, offsets = leaf_lists(nodes, self.x.device)
        d_in, dim, dtype = self.x.shape[1], classes.shape[1], self.x.dtype
        # the gradient steps are taken in 32 bits; the products read copies
        weight = torch.zeros(len(leaves), dim, d_in, device=self.x.device)
        bias = torch.zeros(len(leaves), dim, device=self.x.device)
        y = torch.empty_like(embed)
        for _ in range(steps):
            w, b, c = weight.to(dtype), bias.to(dtype), self.classes
            B.gbdt_leaf_product(self.x, w, offsets, row_idx=row_idx, bias=b, y_out=y)
            h = (self._embed + y).to(dtype)
            loss, lse = B.gbdt_softmax_loss(h, c, self.labels)
            dh, dc = B.gbdt_softmax_grad(h, c, self.labels, lse, scale=1.0 / max(self.counted, 1))
            _, dw, db = B.gbdt_leaf_product_grad(dh, self.x, w, offsets, row_idx=row_idx, want=("weight", "bias"))
            weight -= rate * dw.float()
            bias -= rate * db.float()
            self._classes = self._classes - rate * dc.float()
        w, b = weight.to(dtype), bias.to(dtype)
        self._embed = self._embed + B.gbdt_leaf_product(self.x, w, offsets, row_idx=row_idx, bias=b, y_out=y)
        self.trees.append((nodes, leaves, w, b))
        return self.loss()[0]

    def embed_rows(self, x, bins):
        """Embeddings of other rows (one row is answered as well as many)."""
        h = torch.zeros(x.shape[0], self._classes.shape[1], device=x.device)
        for nodes, leaves, w, b in self.trees:
            row_idx, offsets = route(nodes, bins, leaves)
            h += B.gbdt_leaf_product(x, w, offsets, row_idx=row_idx, bias=b)
        return h.to(x.dtype)

    def probabilities(self, x, bins, class_begin=0, class_end=None):
        """[classes, rows]: the softmax of other rows for a range of classes."""
        h = self.embed_rows(x, bins)
        _, lse = B.gbdt_softmax_loss(h, self.classes)
        end = self.n_classes if class_end is None else class_end
        return B.gbdt_softmax_stats(h, self.classes, None, lse, class_begin, end)[0]


def synthetic(n_rows=20_000, n_features=28, n_classes=500, seed=0, dtype=torch.float32, device="cuda"):
    """Rows whose class follows from which of two halves a feature lies in and from a linear map inside each half."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n_rows, n_features, generator=gen)
    centres = torch.randn(n_classes, 8, generator=gen)
    maps = torch.randn(2, n_features, 8, generator=gen) * n_features ** -0.5
    half = (x[:, 0] > 0).long()
    z = torch.where(half[:, None] > 0, x @ maps[1], x @ maps[0])
    labels = (z @ centres.t()).argmax(1).to(torch.int32)
    edges = torch.linspace(-2.5, 2.5, 63)
    bins = torch.bucketize(x, edges).to(torch.uint8)
    return x.to(dtype).to(device), bins.to(device), 64, labels.to(device), n_classes


def main(trees=8):
    x, bins, n_bins, labels, n_classes = synthetic()
    model = Model(x, bins, n_bins, labels, n_classes, dim=16)
    print("rows %d, classes %d, loss %.4f" % (x.shape[0], n_classes, model.loss()[0]), flush=True)
    for t in range(trees):
        loss = model.add_tree(rate=4.0)
        print("tree %d: %d leaves, loss %.4f" % (t + 1, len(model.trees[-1][1]), loss), flush=True)
    p = model.probabilities(x[:1], bins[:1])
    print("one row: class %d, probability %.3f, label %d" % (int(p[:, 0].argmax()), float(p.max()), int(labels[0])), flush=True)


if __name__ == "__main__":
    main()
