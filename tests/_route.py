"""Routing to experts in 64 bits, from its definition (torch, any device)."""
import math

import torch


def scores(x, score):
    return torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)


def usable(x, score):
    """Rows that have scores."""
    bad = torch.isnan(x).any(1) | (x == -math.inf).all(1)
    return ~(bad | (x == math.inf).any(1)) if score == "softmax" else ~bad


def choose(x, k, score, bias=None, groups=1, kept=1, two=False):
    """ids [N, k] of rows with scores, -1 where too few are left."""
    N, E = x.shape
    x = x.double()
    s = scores(x, score)
    key = x + 0.0 if bias is None else s + bias.double()
    dead = x == -math.inf
    if bias is not None:
        dead = dead | ~(bias > -math.inf)
    key = key.masked_fill(dead, -math.inf)
    if groups > 1 and kept < groups:
        size = E // groups
        by = torch.sort(key.view(N, groups, size), dim=2, descending=True, stable=True)
        value = by.values[:, :, 0]
        if two:
            in_group = torch.gather(s.view(N, groups, size), 2, by.indices) if bias is None else by.values
            first = in_group[:, :, 0].masked_fill(by.values[:, :, 0] == -math.inf, -math.inf)
            second = torch.zeros_like(first) if size == 1 else in_group[:, :, 1].masked_fill(by.values[:, :, 1] == -math.inf, 0.0)
            value = first + second
        best = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :kept]
        stays = torch.zeros(N, groups, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        key = key.masked_fill(~stays.repeat_interleave(size, 1), -math.inf)
    top = torch.sort(key, dim=1, descending=True, stable=True)
    return top.indices[:, :k].masked_fill(top.values[:, :k] == -math.inf, -1).to(torch.int32)


def weights(x, ids, score, renorm, scale, on):
    """Weights [N, k] of ids that may be negative, and their scores."""
    x = x.double()
    there = (ids >= 0) & (ids < x.shape[1]) & on[:, None]
    at = ids.long().clamp(0, x.shape[1] - 1)
    clean = torch.where(on[:, None], x, torch.zeros_like(x))
    s = scores(clean, score).gather(1, at).masked_fill(~there, 0.0)
    if renorm:
        log = (torch.log_softmax(clean, 1) if score == "softmax" else torch.nn.functional.logsigmoid(clean)).gather(1, at)
        log = log.masked_fill(~there, -math.inf)
        best = log.amax(1, keepdim=True)
        e = torch.exp(log - torch.where(best > -math.inf, best, torch.zeros_like(best)))
        s = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    return scale * s


def gradient(x, ids, w, g, score, renorm, scale, on):
    """(gradient [N, E], the sum of its terms' absolute values)"""
    x, g = x.double(), g.double()
    N, E = x.shape
    there = (ids >= 0) & (ids < E) & on[:, None]
    at = ids.long().clamp(0, E - 1)
    clean = torch.where(on[:, None], x, torch.zeros_like(x))
    zero = torch.zeros(N, E, dtype=torch.float64, device=x.device)
    if scale == 0:
        return zero, zero
    g = g.masked_fill(~there, 0.0)
    c, c_size = (g * w).sum(1, keepdim=True), (g * w).abs().sum(1, keepdim=True)
    slope = torch.sigmoid(-clean).gather(1, at) if score == "sigmoid" else torch.ones_like(w)
    if renorm:
        d, size = slope * w * (g - c / scale), slope * w.abs() * (g.abs() + c_size / abs(scale))
    elif score == "sigmoid":
        d, size = slope * w * g, (slope * w * g).abs()
    else:
        s = torch.softmax(clean, 1)
        a = zero.scatter_add(1, at, scale * g)
        any_there = there.any(1, keepdim=True)
        return torch.where(any_there, s * (a - c), zero), s * (a.abs() + c_size)
    d, size = d.masked_fill(~there, 0.0), size.masked_fill(~there, 0.0)
    return zero.scatter_add(1, at, d), zero.scatter_add(1, at, size)
