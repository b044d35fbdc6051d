"""Microscaled 4-bit floats and the balance loss in 64 bits on the CPU, written from their
definitions for the GPU tests (torch, no code of the package)."""
from __future__ import annotations

import math

import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def scale_cols(H):
    return -(-H // 128) * 4


def decode(q, scales, H):
    """Values in double of codes [..., H/2] and scale bytes [..., cols]; NaN for 255."""
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2).long()
    v = MAGNITUDES[code & 7] * torch.where(code > 7, -1.0, 1.0).double()
    s = scales[..., :H // 32].int()
    two = torch.ldexp(torch.ones(s.shape, dtype=torch.float64), s - 127)
    two = torch.where(s == 255, math.nan, two)
    return v * two.repeat_interleave(32, -1)


def quantize(x):
    """Codes [rows, H/2], scale bytes [rows, cols] and values of bf16 rows x."""
    rows, H = x.shape
    b = x.double().view(rows, H // 32, 32)
    a = b.abs().amax(2)
    bad = ~torch.isfinite(b).all(2)
    # the least e with a < 7 * 2^e, found from a's own exponent; at least 2^-127
    mantissa, exponent = torch.frexp(torch.where(bad | (a == 0), 1.0, a))   # in [0.5, 1)
    e = torch.where(mantissa < 0.875, exponent - 3, exponent - 2).clamp(min=-127)
    e = torch.where(a == 0, 0, e)
    unit = torch.ldexp(torch.ones_like(a), e)
    m = torch.where(bad[:, :, None], 0.0, b).abs() / unit[:, :, None]
    far = (m[..., None] - MAGNITUDES).abs()
    near = far.amin(-1, keepdim=True)
    place = torch.arange(8)
    # of two magnitudes equally near the one of even place
    code = torch.where(far == near, place + 8 * (place % 2), 100).amin(-1) % 8
    code = code + torch.where(torch.signbit(b), 8, 0)
    code = code.view(rows, H)
    q = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8)
    scales = torch.zeros(rows, scale_cols(H), dtype=torch.uint8)
    scales[:, :H // 32] = torch.where(bad, 255, e + 127).to(torch.uint8)
    return q, scales, decode(q, scales, H)


def matmul(a, w, windows, swiglu):
    """Products of rows a [rows,K] with w [E,N,K] (double) and what bounds the error of sums in
    float32; rows of no window give NaN.

    A matrix instruction adds 128 products to a running sum; each of the 129 terms may lose
    2^-23 of the largest, which the sum of all magnitudes bounds: 129 / 2^23 of that for each
    instruction."""
    K, out = a.shape[1], w.shape[1] // 2 if swiglu else w.shape[1]
    y = torch.full((a.shape[0], out), math.nan, dtype=torch.float64)
    tol = torch.zeros_like(y)
    step = -(-K // 128) * 129 / 2.0 ** 23
    for e, (s, n) in enumerate(windows):
        rows = a[s:s + n]
        v, t = rows @ w[e].T, rows.abs() @ w[e].abs().T * step
        if swiglu:
            g, u, tg, tu = v[:, :out], v[:, out:], t[:, :out], t[:, out:]
            silu = g * torch.sigmoid(g)
            # |silu'| < 1.1; exp and reciprocal: |g| + 3 units of 2^-23
            tol[s:s + n] = 1.1 * tg * (u.abs() + tu) + silu.abs() * tu \
                + silu.abs() * u.abs() * (g.abs() + 3) * 2.0 ** -23
            v = silu * u
        else:
            tol[s:s + n] = t
        y[s:s + n] = v
    return y, tol


def shares(x, mask, sigmoid):
    """Scores of live tokens over their sum [T,E]; differentiable where x is finite."""
    ok = x > -math.inf
    if mask is not None:
        ok = ok & (mask != 0)[:, None]
    finite = torch.where(ok, x, torch.zeros_like(x))
    if sigmoid:
        v = torch.where(ok, torch.sigmoid(finite), torch.zeros_like(x))
    else:
        top = torch.where(ok, finite.detach(), torch.full_like(x, -1e300)).amax(1, keepdim=True)
        v = torch.where(ok, torch.exp(finite - torch.where(ok.any(1, keepdim=True), top, 0.0)),
                        torch.zeros_like(x))
    t = v.sum(1, keepdim=True)
    return v / torch.where(t > 0, t, torch.ones_like(t))


def balance(x, idx, mask, sigmoid, seq):
    """expert_count, live_tokens, mean_score, loss of logits x [T,E] (double)."""
    T, E = x.shape
    S = T // seq if seq else 1
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask != 0
    use = (idx >= 0) & (idx < E) & live[:, None]
    count = torch.zeros(S, E, dtype=torch.int64)
    for t, j in torch.nonzero(use).tolist():
        count[t // seq if seq else 0, idx[t, j]] += 1
    tokens = live.view(S, -1).sum(1)
    return count, tokens, *losses(x, count, tokens, mask, sigmoid, S)


def losses(x, count, tokens, mask, sigmoid, S):
    E = x.shape[1]
    p = shares(x, mask, sigmoid).reshape(S, -1, E)
    mean = p.sum(1) / tokens.clamp(min=1)[:, None]
    total = count.sum(1, keepdim=True)
    f = count.double() * E / total.clamp(min=1)
    return mean, (f * mean).sum(1)


def balance_grad(x, count, tokens, mask, sigmoid, grad_loss):
    """Gradient of the logits by automatic differentiation, and the size of the terms that
    it is a difference of."""
    S, E = count.shape
    x = x.clone().requires_grad_()
    _, loss = losses(x, count, tokens, mask, sigmoid, S)
    (g,) = torch.autograd.grad((loss * grad_loss).sum(), x)
    p = shares(x.detach(), mask, sigmoid).reshape(S, -1, E)
    f = (count.double() * E / count.sum(1, keepdim=True).clamp(min=1))[:, None]
    size = p * (f + (f * p).sum(2, keepdim=True))
    if sigmoid:
        size = size * torch.sigmoid(-x.detach()).nan_to_num(1.0).reshape(size.shape)
    size = size * (grad_loss.abs() / tokens.clamp(min=1))[:, None, None]
    return torch.where(x > -math.inf, g, torch.zeros_like(g)).detach(), size.reshape(x.shape)
