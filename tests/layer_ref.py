"""The layer's operators in 64 bits on the CPU, written from their definitions
for the GPU tests (torch, no code of the package)."""
from __future__ import annotations

import math

import torch

AMAX_MIN = 2.0 ** -100


def scores(x, sigmoid):
    """Scores of the logits x [T,E] (double); 0 for -inf and NaN."""
    ok = x > -math.inf
    if sigmoid:
        return torch.where(ok, torch.sigmoid(x), torch.zeros_like(x))
    m = torch.where(ok, x, torch.full_like(x, -math.inf)).amax(1, keepdim=True)
    e = torch.where(ok & (x == m), torch.ones_like(x), torch.exp(x - m))
    e = torch.where(ok, e, torch.zeros_like(e))
    t = e.sum(1, keepdim=True)
    return e / torch.where(t > 0, t, torch.ones_like(t))


def keys(x, sigmoid, bias, groups, group_top):
    """Keys in double of every expert, -inf where it is not eligible."""
    k = x.clone()
    if bias is not None or (groups > 1 and group_top > 1):
        k = scores(x, sigmoid) + (0 if bias is None else bias.double())
    return torch.where((x > -math.inf) & (k > -math.inf), k, torch.full_like(k, -math.inf))


def kept_groups(row, groups, top_groups, group_top):
    """Groups of one token's keys (a list) that take part, and the margin to the
    best group left out."""
    size = len(row) // groups
    best = []
    for g in range(groups):
        v = sorted((q for q in row[g * size:(g + 1) * size] if q > -math.inf), reverse=True)
        best.append(sum(v[:group_top]) if v else -math.inf)
    order = sorted(range(groups), key=lambda g: (-best[g], g))
    keep = [g for g in order[:top_groups] if best[g] > -math.inf]
    left = order[len(keep)] if len(keep) < groups else None
    margin = best[keep[-1]] - best[left] if keep and left is not None else math.inf
    return keep, margin


def weights(x, idx, sigmoid, renorm, scale):
    """Weights of the chosen experts idx [T,k] (-1: none)."""
    used = idx >= 0
    at = idx.clamp(min=0).long()
    xc = torch.where(used, x.gather(1, at), torch.full_like(at, 0).double() - math.inf)
    if renorm and not sigmoid:
        m = xc.amax(1, keepdim=True)
        w = torch.where(xc == m, torch.ones_like(xc), torch.exp(xc - m))
    else:
        w = scores(x, sigmoid).gather(1, at)
    w = torch.where(used, w, torch.zeros_like(w))
    if renorm:
        t = w.sum(1, keepdim=True)
        w = w / torch.where(t > 0, t, torch.ones_like(t))
    return w * scale


def route_grad(x, idx, grad_w, sigmoid, renorm, scale):
    """Gradient of the logits by automatic differentiation of `weights`."""
    finite = torch.where(x > -math.inf, x, torch.full_like(x, -1e30)).requires_grad_()
    used = idx >= 0
    at = idx.clamp(min=0).long()
    p = torch.sigmoid(finite) if sigmoid else torch.softmax(finite, 1)
    w = torch.where(used, p.gather(1, at), torch.zeros_like(grad_w))
    if renorm:
        t = w.sum(1, keepdim=True)
        w = w / torch.where(t > 0, t, torch.ones_like(t))
    (g,) = torch.autograd.grad((w * grad_w * scale).sum(), finite)
    return torch.where(x > -math.inf, g, torch.zeros_like(g))


def rmsnorm(x, residual, weight, eps):
    h = x if residual is None else x + residual
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    return h, rstd, h * rstd[:, None] * weight


def amax_scales(v, fp8):
    """Scale of each value of rows v, as a tensor of v's shape."""
    b = v.view(v.shape[0], -1, 128 if fp8 else v.shape[1])
    a = b.abs().amax(2, keepdim=True)
    s = torch.where(a > 0, a.clamp(min=AMAX_MIN) / (448 if fp8 else 127), torch.ones_like(a))
    return s.expand_as(b).reshape(v.shape)


def rmsnorm_grad(grad_y, h, rstd, weight, grad_sum):
    u = grad_y * weight
    r = rstd[:, None]
    dx = r * u - h * r ** 3 * (u * h).mean(1, keepdim=True)
    if grad_sum is not None:
        dx = dx + grad_sum
    return dx, (grad_y * h * r).sum(0)


def expert_matmul(a, a_scale, w, w_scale, windows, swiglu):
    """windows: (first row, rows) of each expert; rows of none give NaN."""
    out = w.shape[1] // 2 if swiglu else w.shape[1]
    y = torch.full((a.shape[0], out), math.nan, dtype=torch.float64)
    for e, (s, n) in enumerate(windows):
        v = (a[s:s + n].double() @ w[e].double().T) * a_scale[s:s + n, None].double() \
            * w_scale[e].double()
        if swiglu:
            g, u = v[:, :out], v[:, out:]
            v = g * torch.sigmoid(g) * u
        y[s:s + n] = v
    return y
