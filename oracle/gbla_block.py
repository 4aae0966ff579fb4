"""64-bit references of the decoder block's operators (torch on the CPU).

``delta`` / ``delta_backward``: the gated delta rule as the recurrence that defines it, token
by token, and its reverse; one sequence at a time, no chunks, everything in float64.
``delta_sizes`` bounds what errors in the terms of a chunked evaluation can add up to.
``add_norm`` / ``add_norm_backward`` / ``to_e4m3``: the residual's addition, the RMS norm over
the width, and rounding to eight bits.
"""
from __future__ import annotations

import torch


def _shared(x, heads):
    """x [H, ..] in 64 bits, each head repeated for the value heads that share it."""
    return x.double().repeat_interleave(heads // x.shape[0], dim=0)


def delta(q, k, v, g, beta, scale, S0=None):
    """q, k [H, n, d], v [V, n, d], g, beta [V, n], S0 [V, d, d] or None -> (out, final state)."""
    V, n, d = v.shape
    q, k, v, beta = _shared(q, V), _shared(k, V), v.double(), beta.double()
    lam = torch.exp(g.double())
    S = torch.zeros(V, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    out = torch.zeros(V, n, d, dtype=torch.float64)
    for t in range(n):
        S = lam[:, t, None, None] * S
        u = beta[:, t, None] * (v[:, t] - torch.matmul(k[:, t, None, :], S)[:, 0])
        S = S + k[:, t, :, None] * u[:, None, :]
        out[:, t] = scale * torch.matmul(q[:, t, None, :], S)[:, 0]
    return out, S


def delta_backward(q, k, v, g, beta, do, scale, S0=None, dS=None):
    """Gradients (dq, dk, dv, dg, dbeta, dS0) of sum(out * do) + sum(final state * dS)."""
    V, n, d = v.shape
    H = q.shape[0]
    q, k, v, beta, do = _shared(q, V), _shared(k, V), v.double(), beta.double(), do.double()
    lam = torch.exp(g.double())
    S = torch.zeros(V, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    past = []
    for t in range(n):
        Z = lam[:, t, None, None] * S
        miss = v[:, t] - torch.matmul(k[:, t, None, :], Z)[:, 0]
        S = Z + k[:, t, :, None] * (beta[:, t, None] * miss)[:, None, :]
        past.append((Z, miss, S))
    D = torch.zeros_like(S) if dS is None else dS.double().clone()
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(v)
    dg, db = torch.zeros_like(beta), torch.zeros_like(beta)
    for t in reversed(range(n)):
        Z, miss, S = past[t]
        o = scale * do[:, t]
        D = D + q[:, t, :, None] * o[:, None, :]
        dq[:, t] = torch.matmul(S, o[:, :, None])[..., 0]
        f = torch.matmul(k[:, t, None, :], D)[:, 0]
        dv[:, t] = beta[:, t, None] * f
        db[:, t] = (f * miss).sum(-1)
        dk[:, t] = (torch.matmul(D, (beta[:, t, None] * miss)[:, :, None])
                    - torch.matmul(Z, dv[:, t, :, None]))[..., 0]
        D = D - k[:, t, :, None] * dv[:, t, None, :]
        dg[:, t] = (D * Z).sum((1, 2))
        D = lam[:, t, None, None] * D
    fold = lambda x: x.view(H, V // H, n, d).sum(1)
    return fold(dq), fold(dk), dv, dg, db, D


def delta_sizes(q, k, v, g, beta, scale, S0=None, tile=64):
    """(out size [V, n, d], state size [V, 1, d]) for keys of length at most one and beta within
    [0, 1].  Then a token's map of the state, exp(g) (I - beta k k^T), makes no column longer, so
    an error in what a token adds to a column stays at most its length, times later decays.
    With norms of a column's vectors over the key channels: a token's error in u is (per unit of
    relative error) at most beta times |v| + the column of the state before its tile + the
    tile's beta |y| and |u| up to it (the first from the product with M, the second as if M,
    which substitution finds, were that of keys whose products are off), where |y| is itself at
    most |v| + that column.  The state's size
    is the decayed sum of those, of |u| and of the state carried over tiles; an output's is
    scale |q| times the state's size, the tile's own column and its |u|."""
    V, n, d = v.shape
    q, k, v, beta = _shared(q, V), _shared(k, V), v.double(), beta.double()
    lam = torch.exp(g.double())[..., None]
    S = torch.zeros(V, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    norm = lambda X: X.norm(dim=1)
    Z = norm(S)
    out = torch.zeros(V, n, d, dtype=torch.float64)
    for t in range(n):
        if t % tile == 0:
            head, inner, added = norm(S), torch.zeros(V, d), torch.zeros(V, d)
            Z = Z + head
        S = lam[:, t, :, None] * S
        u = beta[:, t, None] * (v[:, t] - torch.matmul(k[:, t, None, :], S)[:, 0])
        S = S + k[:, t, :, None] * u[:, None, :]
        y = v[:, t].abs() + head
        inner, added = inner + beta[:, t, None] * y, added + u.abs()
        Z = lam[:, t] * Z + beta[:, t, None] * (y + inner + added) + u.abs()
        out[:, t] = abs(scale) * q[:, t].norm(dim=-1, keepdim=True) * (Z + head + added)
    return out, Z[:, None, :]


def delta_backward_sizes(q, k, v, g, beta, do, scale, S0=None, dS=None, tile=64):
    """The like of ``delta_sizes`` for (dq, dk, dv, dg, dbeta, dS0).  A token's map of the state's
    gradient is the transpose of the forward's and makes no column longer either, so of an error
    in f = D^T k only what arises at the token adds to W, the error that the state's gradient
    carries.  Per token and value channel: A bounds an error in reading the state, Bu one in u, G
    one in reading the state's gradient, Bf one in f (from the tile's do, the gradient after the
    tile and the tile's later f).  dk = D u - Z dv takes both factors' errors of both products,
    dbeta = f miss likewise; dg adds up, over the sequence, those of what a token's do and dv take of the
    past (the state before its tile and the tile's earlier u) and of what its u gives to the
    gradient after the tile, and of one <D, S>, the largest of those where tiles meet."""
    V, n, d = v.shape
    H = q.shape[0]
    q, k, v, beta, do = _shared(q, V), _shared(k, V), v.double(), beta.double(), do.double()
    lam = torch.exp(g.double())[..., None]
    norm = lambda X: X.norm(dim=1)
    S = torch.zeros(V, d, d, dtype=torch.float64) if S0 is None else S0.double().clone()
    Z = norm(S)
    past, starts = [], {}
    for t in range(n):
        if t % tile == 0:
            starts[t] = (norm(S), Z)
            head, inner, added = norm(S), torch.zeros(V, d), torch.zeros(V, d)
            Z = Z + head
        P = lam[:, t, :, None] * S
        miss = v[:, t] - torch.matmul(k[:, t, None, :], P)[:, 0]
        u = beta[:, t, None] * miss
        S = P + k[:, t, :, None] * u[:, None, :]
        y = v[:, t].abs() + head
        reach = head + added  # of what the token's key finds
        inner, added = inner + beta[:, t, None] * y, added + u.abs()
        wrong = Z + y + inner + added  # of miss
        Z = lam[:, t] * Z + beta[:, t, None] * (y + inner + added) + u.abs()
        past.append((P, miss, u, S, Z + head + added, wrong, reach))
    D = torch.zeros_like(S) if dS is None else dS.double().clone()
    W = norm(D)
    out = {x: torch.zeros(V, n, d, dtype=torch.float64) for x in ("dq", "dk", "dv")}
    db = torch.zeros(V, n, dtype=torch.float64)
    flow = torch.zeros(V, dtype=torch.float64)
    meet = (norm(S) * W + Z * norm(D)).sum(-1)
    for t in reversed(range(n)):
        if t == n - 1 or t % tile == tile - 1:
            tail, given, later = norm(D), torch.zeros(V, d), torch.zeros(V, d)
            W = W + tail
        P, miss, u, S, A, wrong, reach = past[t]
        o = abs(scale) * do[:, t].abs()
        D = D + scale * q[:, t, :, None] * do[:, t, None, :]
        f = torch.matmul(k[:, t, None, :], D)[:, 0]
        dv = beta[:, t, None] * f
        given = given + o
        W = W + q[:, t].norm(dim=-1, keepdim=True) * o
        near = tail + given + later
        G = W + near
        near = near + beta[:, t, None] * (tail + given)
        Bf = W + near
        later = later + dv.abs() + beta[:, t, None] * (tail + given)
        out["dq"][:, t] = (A * o).sum(-1, keepdim=True)
        out["dv"][:, t] = beta[:, t, None] * Bf
        Bu = beta[:, t, None] * wrong
        out["dk"][:, t] = (G * u.abs() + (norm(D) + tail + given + later) * Bu + A * dv.abs()
                           + (norm(P) + A) * out["dv"][:, t]).sum(-1, keepdim=True)
        db[:, t] = (Bf * miss.abs() + f.abs() * wrong).sum(-1)
        flow = flow + (A * o + dv.abs() * wrong + out["dv"][:, t] * reach + u.abs() * (W + tail) + tail * Bu).sum(-1)
        D = D - k[:, t, :, None] * dv[:, None, :]
        W = lam[:, t] * (W + beta[:, t, None] * near + dv.abs())
        D = lam[:, t, :, None] * D
        if t in starts:
            meet = torch.maximum(meet, (starts[t][0] * W + starts[t][1] * norm(D)).sum(-1))
    dg = (flow + meet)[:, None]
    fold = lambda x: x.view(H, V // H, n, d).sum(1)
    return fold(out["dq"]), fold(out["dk"]), out["dv"], dg.expand(V, n), db, W[:, None, :].expand(V, d, d)


def add_norm(x, residual, w, eps):
    """(normalised, sum): the sum rounded to x's type, and the norm of that sum."""
    s = x.double() if residual is None else (x.double() + residual.double()).to(x.dtype).double()
    return s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * w.double(), s


def add_norm_backward(s, w, dy, ds, eps):
    """(dx, dw) of sum(normalised * dy) + sum(sum * ds)."""
    s, dy, w = s.double(), dy.double(), w.double()
    r = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    n, u = s * r, dy * w
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    return (dx if ds is None else dx + ds.double()), (dy * n).reshape(-1, s.shape[-1]).sum(0)


def to_e4m3(x):
    """x rounded to four bits of exponent and three of fraction: half to even, steps of 2^-9
    below 2^-6, at most 448."""
    x = x.double()
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp(min=-9))
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)
