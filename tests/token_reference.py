"""The operators on a token's way in 64 bits, from their definitions: row by row and without the library."""
import math

import numpy as np
import torch

D = torch.float64


def route(z, bias, k, scores="softmax", groups=1, kept=1, best=1, renormalise=True, scale=1.0):
    """(experts, weights) of one row: z a list of numbers, bias such a list or None."""
    E = len(z)
    b = [0.0] * E if bias is None else list(bias)
    if any(math.isnan(x) or (scores == "softmax" and x == math.inf) for x in z) or any(math.isnan(x) or x == math.inf for x in b):
        return list(range(k)), [math.nan] * k
    open_ = [z[e] > -math.inf and b[e] > -math.inf for e in range(E)]
    s = score(z, scores)
    v = [s[e] + b[e] for e in range(E)] if bias is not None else s
    allowed = list(open_)
    if groups > 1:
        size = E // groups
        total = []
        for g in range(groups):
            mine = sorted((v[e] if bias is not None or best > 1 else z[e] for e in range(g * size, (g + 1) * size) if open_[e]), reverse=True)[:best]
            total.append(sum(mine) if mine else -math.inf)
        ranked = sorted(range(groups), key=lambda g: (-total[g], g))[:kept]
        allowed = [open_[e] and e // size in ranked for e in range(E)]
    order = sorted((e for e in range(E) if allowed[e]), key=lambda e: (-(v[e] if bias is not None else z[e]), e))[:k]
    chosen = [s[e] for e in order]
    if renormalise and order:
        if scores == "softmax":
            top = max(z[e] for e in order)
            chosen = [math.exp(z[e] - top) for e in order]
        elif max(z[e] for e in order) < 0:                  # scores over e^top, top < 0
            top = max(z[e] for e in order)
            chosen = [math.exp(z[e] - top) / (1 + math.exp(z[e])) for e in order]
        chosen = [x / sum(chosen) for x in chosen]
    missing = k - len(order)
    return order + [-1] * missing, [scale * x for x in chosen] + [0.0] * missing


def score(z, scores):
    if scores == "sigmoid":
        return [1 / (1 + math.exp(-x)) if x > -700 else 0.0 for x in z]
    top = max(z)
    if top == -math.inf:
        return [0.0] * len(z)
    t = [math.exp(x - top) for x in z]
    return [x / sum(t) for x in t]


def weights_of(z, experts, scores, renormalise, scale):
    """Weights of given experts as a function of the logits, differentiable: z [rows][E] in 64 bits, experts [rows][k] with -1."""
    there = experts >= 0
    at = experts.clamp(min=0).long()
    s = torch.softmax(z, 1) if scores == "softmax" else torch.sigmoid(z)
    s = torch.where(there, s.gather(1, at), 0)
    if renormalise:
        s = s / torch.where(there.any(1, keepdim=True), s.sum(1, keepdim=True), 1)
    return scale * s


def order(experts, first, E):
    """(offsets, places) by counting, entry by entry."""
    flat = experts.reshape(-1).astype(np.int64) - first
    mine = (flat >= 0) & (flat < E)
    load = np.bincount(flat[mine], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(load)])
    places = np.full(flat.size, -1, np.int64)
    at = np.argsort(np.where(mine, flat, E), kind="stable")[:int(mine.sum())]
    places[at] = np.arange(at.size)
    return offsets, places.reshape(experts.shape)


def norm(x, w, b, eps, centred):
    """(y, mean, rstd), differentiable."""
    mean = x.mean(1) if centred else torch.zeros_like(x[:, 0])
    d = x - mean.unsqueeze(1)
    rstd = 1 / torch.sqrt((d * d).mean(1) + eps)
    y = d * rstd.unsqueeze(1)
    if w is not None:
        y = y * w
    return (y + b if b is not None else y), mean, rstd


def norm_gradients(dy, x, w, mean, rstd, centred):
    """(dx, dw, db) by the formula."""
    xh = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
    g = dy * w if w is not None else dy
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if centred:
        dx = dx - g.mean(1, keepdim=True)
    return dx * rstd.unsqueeze(1), (dy * xh).sum(0), dy.sum(0)


def route_gradients(z, experts, g, scores, renormalise, scale):
    """dz by the formulas."""
    there = experts >= 0
    at = experts.clamp(min=0).long()
    s = torch.softmax(z, 1) if scores == "softmax" else torch.sigmoid(z)
    s = torch.where(torch.isnan(s), torch.zeros_like(s), s)             # (rows whose logits are all -inf)
    c, g = torch.where(there, s.gather(1, at), 0), torch.where(there, g, 0)
    if renormalise:
        p = c / torch.where(c.sum(1, keepdim=True) > 0, c.sum(1, keepdim=True), 1)
        d = scale * p * (g - (g * p).sum(1, keepdim=True)) * (1 - c if scores == "sigmoid" else 1)
        return torch.zeros_like(z).scatter_add_(1, at, torch.where(there, d, 0))
    if scores == "sigmoid":
        return torch.zeros_like(z).scatter_add_(1, at, scale * g * c * (1 - c))
    full = torch.zeros_like(z).scatter_add_(1, at, g)
    return scale * s * (full - (g * c).sum(1, keepdim=True))
