"""Routing of rows to several linear leaves, weighted products and 8-bit codes from their definitions, in 64 bits, with torch on
whichever device the inputs are on.  Shares nothing with the HIP library.  Functions that a rounding analysis needs sums of
magnitudes for return them as well."""
from __future__ import annotations

import torch

F64, LOW = torch.float64, float("-inf")


def scores(logits, score):
    """64-bit scores; masked logits (NaN, minus infinity) have none: 0."""
    l = logits.double()
    l = torch.where(torch.isnan(l), torch.full_like(l, LOW), l)
    if score == "sigmoid":
        return torch.where(l == LOW, 0.0, torch.sigmoid(l)), l
    top = l.amax(1, keepdim=True)
    e = torch.where(l == top, 1.0, torch.exp(l - top))
    e = torch.where(l == LOW, 0.0, e)
    return e / e.sum(1, keepdim=True).clamp(min=1e-300), l


def route(logits, k, choice_bias=None, score="softmax", n_groups=1, groups_kept=1, group_best=1, renormalise=True, scale=1.0):
    """(leaves int32, gates float64)."""
    s, l = scores(logits, score)
    n, n_leaves = l.shape
    c = l if choice_bias is None else s + choice_bias.double()  # what leaves are chosen by
    v = s if choice_bias is None and group_best == 2 else c      # what groups are worth
    c, v = (torch.where((l == LOW) | torch.isnan(c), torch.full_like(c, LOW), t) for t in (c, v))
    if n_groups > 1:
        g = v.view(n, n_groups, -1)
        best = torch.sort(g, dim=2, descending=True)[0][:, :, :group_best]
        worth = torch.where(best[:, :, 0] == LOW, best[:, :, 0], torch.where(best == LOW, 0.0, best).sum(2))
        order = torch.sort(worth, dim=1, descending=True, stable=True)[1][:, :groups_kept]
        keep = torch.zeros_like(worth, dtype=torch.bool).scatter_(1, order, True)
        c = torch.where(keep[:, :, None], c.view(n, n_groups, -1), LOW).reshape(n, n_leaves)
    top, at = torch.sort(c, dim=1, descending=True, stable=True)
    top, at = top[:, :k], at[:, :k]
    leaves = torch.where(top == LOW, -1, at).to(torch.int32)
    return leaves, weights(logits, leaves, score, renormalise, scale)


def _chosen(logits, leaves, score, renormalise):
    """(use, scores of the slots or their shares, what 1 - score is)."""
    s, l = scores(logits, score)
    use = (leaves >= 0) & (leaves < logits.shape[1])
    at = torch.where(use, leaves, 0).long()
    at_l = l.gather(1, at)
    use = use & (at_l > LOW)
    if not renormalise:
        return use, torch.where(use, s.gather(1, at), 0.0), at_l
    # shares from logarithms, so that they hold where all scores vanish
    ls = at_l if score == "softmax" else torch.nn.functional.logsigmoid(at_l)
    ls = torch.where(use, ls, LOW)
    top = ls.amax(1, keepdim=True)
    e = torch.where(use, torch.where(ls == top, 1.0, torch.exp(ls - top)), 0.0)
    return use, e / e.sum(1, keepdim=True).clamp(min=1e-300), at_l


def weights(logits, leaves, score, renormalise, scale):
    return scale * _chosen(logits, leaves, score, renormalise)[1]


def route_grad(logits, leaves, dgates, score="softmax", renormalise=True, scale=1.0):
    """(dlogits, magnitude), float64."""
    use, r, at_l = _chosen(logits, leaves, score, renormalise)
    dg = torch.where(use, dgates.double(), 0.0)
    at = torch.where(use, leaves, 0).long()
    inner, inner_mag = (r * dg).sum(1, keepdim=True), (r * dg).abs().sum(1, keepdim=True)
    out = torch.zeros(logits.shape, dtype=F64, device=logits.device)
    mag = torch.zeros_like(out)
    each, each_mag = scale * r * dg, abs(scale) * r * dg.abs()
    if renormalise:
        each, each_mag = each - scale * r * inner, each_mag + abs(scale) * r * inner_mag
    elif score == "softmax":
        s, _ = scores(logits, score)
        out, mag = -scale * s * inner, abs(scale) * s * inner_mag
    if score == "sigmoid":
        each, each_mag = (v * torch.sigmoid(-at_l) for v in (each, each_mag))
    zero = torch.zeros_like(each)
    out.scatter_add_(1, at, torch.where(use, each, zero))
    mag.scatter_add_(1, at, torch.where(use, each_mag, zero))
    return out, mag


def slots_of(leaves, n_leaves):
    """[(leaf, rows, slots)]."""
    return [(leaf,) + torch.nonzero(leaves == leaf, as_tuple=True) for leaf in range(n_leaves)]


def mixture(x, weight, bias, leaves, gates):
    """(y, magnitude)."""
    n, (n_leaves, d_out, d_in) = x.shape[0], weight.shape
    y = torch.zeros(n, d_out, dtype=F64, device=x.device)
    mag = torch.zeros_like(y)
    for leaf, d, j in slots_of(leaves, n_leaves):
        if d.numel() == 0:
            continue
        a, w, g = x[d].double(), weight[leaf].double().t().contiguous(), gates[d, j].double()[:, None]
        b = torch.zeros(d_out, dtype=F64, device=x.device) if bias is None else bias[leaf].double()
        y.index_add_(0, d, g * (a @ w + b))
        mag.index_add_(0, d, g.abs() * (a.abs() @ w.abs() + b.abs()))
    return y, mag


def mixture_grad(dy, x, weight, bias, leaves, gates):
    """((dx, dweight, dbias, dgates), their magnitudes)."""
    n, (n_leaves, d_out, d_in) = x.shape[0], weight.shape
    shapes = [(n, d_in), tuple(weight.shape), (n_leaves, d_out), tuple(leaves.shape)]
    out = [torch.zeros(s, dtype=F64, device=x.device) for s in shapes]
    mag = [torch.zeros_like(o) for o in out]
    for leaf, d, j in slots_of(leaves, n_leaves):
        if d.numel() == 0:
            continue
        a, w, g = x[d].double(), weight[leaf].double(), gates[d, j].double()[:, None]
        of = dy[d].double()
        b = torch.zeros(d_out, dtype=F64, device=x.device) if bias is None else bias[leaf].double()
        gd = g * of
        out[0].index_add_(0, d, gd @ w)
        mag[0].index_add_(0, d, gd.abs() @ w.abs())
        out[1][leaf], mag[1][leaf] = gd.t().contiguous() @ a, gd.abs().t().contiguous() @ a.abs()
        out[2][leaf], mag[2][leaf] = gd.sum(0), gd.abs().sum(0)
        wt = w.t().contiguous()
        out[3][d, j] = ((a @ wt + b) * of).sum(1)
        mag[3][d, j] = ((a.abs() @ wt.abs() + b.abs()) * of.abs()).sum(1)
    return tuple(out), tuple(mag)


def quantize(x):
    """(codes int8, scales float32): scale = max |x| times the 32-bit 1 / 127, rounded to 32 bits; codes round to even."""
    most = x.float().abs().amax(1)
    finite = torch.isfinite(x.float()).all(1)
    scales = (most.double() * torch.tensor(1.0 / 127.0, dtype=torch.float32).double().item()).float()
    scales = torch.where(scales < 2.0 ** -126, 0.0, scales)
    unit = torch.where(finite & (scales > 0), scales, 1.0).double()
    codes = torch.where((finite & (scales > 0))[:, None], torch.round(x.double() / unit[:, None]), 0.0)
    return codes.to(torch.int8), torch.where(finite, scales, float("nan"))


def padded(codes):
    out = torch.zeros(codes.shape[0], (codes.shape[1] + 15) // 16 * 16, dtype=torch.int8, device=codes.device)
    out[:, :codes.shape[1]] = codes
    return out
