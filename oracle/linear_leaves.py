"""Linear leaves and the softmax over many classes from their definitions, in 64 bits, with torch on whichever device
the inputs are on.  Shares nothing with the HIP library; every function also returns the sums of magnitudes that a
rounding analysis of the 32-bit sums needs."""
from __future__ import annotations

import torch


def leaf_of_rows(offsets, row_idx, n_rows):
    """[(leaf, rows)] with positions outside the list and row ids outside the matrix left out."""
    offsets = [int(o) for o in offsets]
    n = n_rows if row_idx is None else row_idx.numel()
    ids = torch.arange(n) if row_idx is None else row_idx.detach().cpu().long()
    out = []
    for leaf in range(len(offsets) - 1):
        a, b = (min(max(o, 0), n) for o in offsets[leaf:leaf + 2])
        rows = ids[a:b]
        out.append((leaf, rows[(rows >= 0) & (rows < n_rows)]))
    return out


def leaf_product(x, weight, bias, offsets, row_idx, y0):
    """(y, magnitude): y0 with the rows of the leaves overwritten."""
    y, mag = y0.double().clone(), torch.zeros_like(y0, dtype=torch.float64)
    for leaf, rows in leaf_of_rows(offsets, row_idx, x.shape[0]):
        if rows.numel() == 0:
            continue
        rows = rows.to(x.device)
        a, w = x[rows].double(), weight[leaf].double().t().contiguous()
        b = torch.zeros(w.shape[1], dtype=torch.float64, device=x.device) if bias is None else bias[leaf].double()
        y[rows] = a @ w + b
        mag[rows] = a.abs() @ w.abs() + b.abs()
    return y, mag


def leaf_product_grad(dy, x, weight, offsets, row_idx, dx0):
    """((dx, dweight, dbias), their magnitudes)."""
    f64 = torch.float64
    dx, dx_mag = dx0.double().clone(), torch.zeros_like(dx0, dtype=f64)
    dw, dw_mag = torch.zeros_like(weight, dtype=f64), torch.zeros_like(weight, dtype=f64)
    db = torch.zeros(weight.shape[:2], dtype=f64, device=x.device)
    db_mag = torch.zeros_like(db)
    for leaf, rows in leaf_of_rows(offsets, row_idx, x.shape[0]):
        if rows.numel() == 0:
            continue
        rows = rows.to(x.device)
        g, a, w = dy[rows].double(), x[rows].double(), weight[leaf].double()
        dx[rows], dx_mag[rows] = g @ w, g.abs() @ w.abs()
        gt = g.t().contiguous()
        dw[leaf], dw_mag[leaf] = gt @ a, gt.abs() @ a.abs()
        db[leaf], db_mag[leaf] = g.sum(0), g.abs().sum(0)
    return (dx, dw, db), (dx_mag, dw_mag, db_mag)


def scores(h, classes):
    ct = classes.double().t().contiguous()
    return h.double() @ ct, h.double().abs() @ ct.abs()


def counted(labels, n_rows, n_classes, device):
    if labels is None:
        return torch.ones(n_rows, dtype=torch.bool, device=device)
    return (labels >= 0) & (labels < n_classes)


def softmax_loss(h, classes, labels):
    """(loss, lse); rows that do not count are zeros, loss is None without labels."""
    s, _ = scores(h, classes)
    use = counted(labels, h.shape[0], classes.shape[0], h.device)
    lse = torch.logsumexp(s, 1)
    zero = torch.zeros_like(lse)
    if labels is None:
        return None, lse
    picked = s.gather(1, torch.where(use, labels, torch.zeros_like(labels)).long()[:, None])[:, 0]
    return torch.where(use, lse - picked, zero), torch.where(use, lse, zero)


def score_gradient(h, classes, labels, lse, row_weight):
    """G = w (p - [v = y]) from the given lse, zeros for rows that do not count."""
    s, _ = scores(h, classes)
    use = counted(labels, h.shape[0], classes.shape[0], h.device)
    p = torch.exp(s - lse.double()[:, None])
    if labels is not None:
        at = torch.arange(h.shape[0], device=h.device)[use]
        p[at, labels[use].long()] -= 1.0
    w = torch.ones(h.shape[0], dtype=torch.float64, device=h.device) if row_weight is None else row_weight.double()
    return torch.where(use[:, None], p * w[:, None], torch.zeros_like(p))


def softmax_grad(h, classes, labels, lse, row_weight, scale):
    """(dh, dclasses), magnitudes |scale| |G| |C| and |scale| |G|^T |H|."""
    g = score_gradient(h, classes, labels, lse, row_weight)
    use = counted(labels, h.shape[0], classes.shape[0], h.device)
    hs = torch.where(use[:, None], h.double(), torch.zeros_like(h, dtype=torch.float64))
    c, gt = classes.double(), g.t().contiguous()
    return (scale * (g @ c), scale * (gt @ hs)), (abs(scale) * (g.abs() @ c.abs()), abs(scale) * (gt.abs() @ hs.abs()))


def softmax_stats(h, classes, labels, lse, begin, end):
    """(grad, hess), a row a class."""
    s, _ = scores(h, classes[begin:end])
    use = counted(labels, h.shape[0], classes.shape[0], h.device)[:, None]
    p = torch.where(use, torch.exp(s - lse.double()[:, None]), torch.zeros_like(s))
    grad = p.clone()
    if labels is not None:
        grad -= (labels[:, None].long() == torch.arange(begin, end, device=h.device)[None, :]).double()
    return grad.t().contiguous(), (p * (1.0 - p)).t().contiguous()
