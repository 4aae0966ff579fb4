"""64-bit references of the decoder's operators, token by token (torch on the CPU).

``rope`` / ``rope_backward``: the RMS norm of queries or keys and the rotation by
position.  ``decay`` / ``decay_backward``: causal linear attention with a decay per key
head, as the recurrence that defines it and its reverse.  One sequence at a time, no
chunks, no splits; everything in float64.

``decay_sizes`` / ``decay_backward_sizes``: the same sums with every term's absolute
value, which bound what roundings can add up to.
"""
from __future__ import annotations

import torch


def _pairs(d: int, rotary: int, adjacent: bool):
    """(first channels, second channels) of the rotating pairs."""
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rotary // 2)


def _turn(x, positions, rotary, theta, adjacent, sign):
    """x [H, n, d] with each pair turned by sign * position * theta^(-2i/rotary)."""
    y = x.clone()
    if rotary == 0:
        return y
    a, b = _pairs(x.shape[-1], rotary, adjacent)
    angle = positions.double()[:, None] * theta ** (-2.0 * torch.arange(rotary // 2).double() / rotary)
    c, s = torch.cos(angle), sign * torch.sin(angle)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def rope(x, w, positions, rotary, theta=10000.0, eps=1e-6, adjacent=False):
    """x [H, n, d], w [H, d] or None (no norm), positions [n]."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()[:, None, :]
    return _turn(x, positions, rotary, theta, adjacent, 1.0)


def rope_backward(x, w, positions, dy, rotary, theta=10000.0, eps=1e-6, adjacent=False):
    """(dx, dw) of sum(rope * dy); dw None without w."""
    x, u = x.double(), _turn(dy.double(), positions, rotary, theta, adjacent, -1.0)
    if w is None:
        return u, None
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xn = x * r
    uw = u * w.double()[:, None, :]
    return r * (uw - xn * (uw * xn).mean(-1, keepdim=True)), (u * xn).sum(1)


def _decays(g):
    return torch.exp(g.double())[:, None, None]


def decay(q, k, v, g, scale, S0=None):
    """q [H, n, d], k, v [K, n, d], g [K], S0 [K, d, d] or None -> (out, final state)."""
    q, k, v = q.double(), k.double(), v.double()
    (H, n, d), K = q.shape, k.shape[0]
    lam = _decays(g)
    S = torch.zeros(K, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    out = torch.zeros(H, n, d, dtype=torch.float64)
    for t in range(n):
        S = lam * S + k[:, t, :, None] * v[:, t, None, :]
        out[:, t] = scale * torch.matmul(q[:, t].view(K, H // K, d), S).view(H, d)
    return out, S


def decay_backward(q, k, v, g, do, scale, S0=None, dS=None):
    """Gradients (dq, dk, dv, dg, dS0) of sum(out * do) + sum(final state * dS)."""
    q, k, v, do = q.double(), k.double(), v.double(), do.double()
    (H, n, d), K = q.shape, k.shape[0]
    lam = _decays(g)
    S = torch.zeros(K, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    before = []
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(n):
        before.append(S)
        S = lam * S + k[:, t, :, None] * v[:, t, None, :]
        dq[:, t] = scale * torch.matmul(do[:, t].view(K, H // K, d), S.transpose(1, 2)).view(H, d)
    D = torch.zeros_like(S) if dS is None else dS.double().clone()
    dg = torch.zeros(K, dtype=torch.float64)
    for t in reversed(range(n)):
        D = D + scale * torch.matmul(q[:, t].view(K, H // K, d).transpose(1, 2).contiguous(),
                                     do[:, t].view(K, H // K, d))
        dk[:, t] = torch.matmul(D, v[:, t, :, None])[..., 0]
        dv[:, t] = torch.matmul(D.transpose(1, 2), k[:, t, :, None])[..., 0]
        dg += (lam * before[t] * D).sum((1, 2))
        D = lam * D
    return dq, dk, dv, dg, D


def decay_sizes(q, k, v, g, scale, S0=None):
    """``decay`` with every term's absolute value."""
    return decay(q.abs(), k.abs(), v.abs(), g, abs(scale), None if S0 is None else S0.abs())


def decay_backward_sizes(q, k, v, g, do, scale, S0=None, dS=None):
    """``decay_backward`` with every term's absolute value.  The entry for g also counts
    each pair's weight with the largest distance that its rounding can be multiplied by
    (512 tokens, the kernels' longest unit) where that is more than its own."""
    a = lambda x: None if x is None else x.abs()
    dq, dk, dv, dg, dS0 = decay_backward(a(q), a(k), a(v), g, a(do), abs(scale), a(S0), a(dS))
    pairs = (a(k).double() * dk).sum((1, 2))
    return dq, dk, dv, dg + 512.0 * pairs, dS0
