"""Performance cases of the decoder block's operators: the gated delta rule, and the RMS norm
that joins the residual stream, over the sizes that their users run.

In the order a decoder block calls them:

``gbla.add_rms_norm``      the residual's addition and the RMS norm over the width, in the
                           activations' type; ``gbla.add_rms_norm_e4m3`` with an output of
                           8 bits and its scales; ``gbla.add_rms_norm_backward``
``gbla.delta_attention``   the gated delta rule in chunks (prompts, training), and
                           ``gbla.delta_attention_backward``
``gbla.delta_step``        the same rule for one new token of each row of a batch, reading
                           and updating the states

The listed cases take the repository's own workloads (``paper_2606_07317_amd/inputs.py``,
``perf/cases.py``): heads, head dims, the layer's width, lengths, packed batches.  ``draw``
gives further cases of the same ranges: every head dim, both data types, value heads that
share queries and keys, odd lengths, widths and row counts.

A case is a dict of plain values:
  kind      "delta", "delta_bwd", "delta_step", "norm" or "norm_bwd"
  layout    "dense" (batch x seqlen) or "ragged" (batch sequences whose lengths are
            lognormal(len_mu, len_sigma) within [len_min, len_max])
  heads (of q and k), value_heads, head_dim, dtype ("bf16" / "f32")
  state     an initial state is given and the final one returned (delta, delta_bwd)
  slots     delta_step only: states held, of which the batch's rows name some
  lengths_seed  ragged only: seeds the lengths, so that a case's size (and so its work) does
            not change with the seed of its inputs
  rows, width, residual (added before the norm), bits8 (output in 8 bits), group (channels
            of a scale; 0: one scale a row)

With ``own`` false, ``run`` computes the operators from elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6


def listed():
    return [
        # A short full-precision prompt with two heads (the size of the workload tiny_f32, and
        # one token past a round length).
        _delta("delta_f32_b1_n257_h2_d32", "delta", 1, 257, 2, 2, 32, dtype="f32"),
        # One long prompt (the throughput workload's size), whose state the single tokens
        # that follow start from.
        _delta("delta_bf16_b1_n32768_h8_d64", "delta", 1, 32768, 8, 8, 64),
        # Packed prompts of very different lengths that go on from earlier states, wide heads,
        # two value heads to a query and key head.
        _ragged(_delta("delta_bf16_ragged64_h4_v8_d128", "delta", 64, 0, 4, 8, 128, state=True),
                7.5, 1.0, 16, 32768),
        # A training batch's gradients.
        _delta("delta_bwd_bf16_b8_n2048_h16_d64", "delta_bwd", 8, 2048, 16, 16, 64),
        # ... of a packed batch with wide heads, from states and with gradients of the states.
        _ragged(_delta("delta_bwd_bf16_ragged16_h4_v8_d128", "delta_bwd", 16, 0, 4, 8, 128,
                       state=True), 7.5, 1.0, 16, 32768),
        # One token of one sequence: launches and host time are all there is.
        _step("delta_step_bf16_n1_h8_d64", 1, 1, 8, 8, 64),
        # A large serving batch with wide heads, two value heads to a key head, whose states
        # lie among more.
        _step("delta_step_bf16_n256_h4_v8_d128", 256, 320, 4, 8, 128),
        # One new token of four sequences, at the layer's width.
        _norm("norm_bf16_n4_w1024", "norm", 4, 1024),
        # A long prompt's tokens before a projection in 8 bits, a scale for 128 channels.
        _norm("norm_e4m3_n32768_w1024", "norm", 32768, 1024, bits8=True, group=128),
        # A full-precision batch of odd size.
        _norm("norm_f32_n5001_w1288", "norm", 5001, 1288, dtype="f32"),
        # A training batch's gradients (8 x 2048 tokens at the layer's width).
        _norm("norm_bwd_bf16_n16384_w1024", "norm_bwd", 16384, 1024),
        # ... of a wide model in full precision, with an odd number of rows.
        _norm("norm_bwd_f32_n4097_w4096", "norm_bwd", 4097, 4096, dtype="f32"),
    ]


def draw(rng):
    # The kinds in the shares of the listed cases; sizes uniform in their logarithm, from the
    # smallest listed to no more work than the largest.
    kind = rng.choice(["delta"] * 3 + ["delta_bwd"] * 3 + ["delta_step"] * 2 + ["norm"] * 2 + ["norm_bwd"] * 2)
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if kind in ("norm", "norm_bwd"):
        width = 8 * _log_int(rng, 4, 2048)
        rows = _log_int(rng, 1, 2 ** 25 // width)
        bits8 = kind == "norm" and rng.random() < 0.4
        group = 128 if bits8 and width % 128 == 0 and rng.random() < 0.5 else 0
        residual = kind == "norm_bwd" or rng.random() < 0.8
        return _unnamed(_norm(None, kind, rows, width, dtype, residual, bits8, group))
    d = rng.choice([32, 64, 64, 128])
    heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    values = heads * rng.choice([1, 1, 2, 4] if heads <= 4 else [1, 1, 2] if heads == 8 else [1])
    if kind == "delta_step":
        # up to the states of the largest listed case
        rows = _log_int(rng, 1, min(512, 2 ** 25 // (values * d * d)))
        return _unnamed(_step(None, rows, rows + rng.randrange(64), heads, values, d, dtype))
    # up to the tokens of one long prompt for eight heads of 64
    top = {"delta": 2 ** 24, "delta_bwd": 2 ** 23}[kind]
    tokens = _log_int(rng, 16, top // (values * d))
    batch = min(tokens, _log_int(rng, 1, 64))
    case = _delta(None, kind, batch, max(1, tokens // batch), heads, values, d, dtype, rng.random() < 0.5)
    if batch > 1 and rng.random() < 0.5:
        mean, sigma = max(2.0, tokens / batch), rng.choice([0.5, 1.0])
        case = _ragged(case, math.log(mean) - sigma * sigma / 2, sigma, 1,
                       max(16, int(4 * mean)), rng.randrange(1 << 20))
    return _unnamed(case)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _unnamed(case):
    return {n: x for n, x in case.items() if n != "name"}


def _delta(name, kind, batch, seqlen, heads, value_heads, d, dtype="bf16", state=False):
    return dict(name=name, kind=kind, layout="dense", batch=batch, seqlen=seqlen, heads=heads,
                value_heads=value_heads, head_dim=d, dtype=dtype, state=state)


def _step(name, rows, slots, heads, value_heads, d, dtype="bf16"):
    return dict(name=name, kind="delta_step", layout="dense", batch=rows, seqlen=1, slots=slots,
                heads=heads, value_heads=value_heads, head_dim=d, dtype=dtype)


def _norm(name, kind, rows, width, dtype="bf16", residual=True, bits8=False, group=0):
    return dict(name=name, kind=kind, rows=rows, width=width, dtype=dtype, residual=residual,
                bits8=bits8, group=group)


def _ragged(case, mu, sigma, lo, hi, lengths_seed=4):
    return dict(case, layout="ragged", seqlen=0, len_mu=mu, len_sigma=sigma, len_min=lo, len_max=hi,
                lengths_seed=lengths_seed)


def _lengths(case):
    """Length of every sequence of the batch."""
    if case["layout"] == "dense":
        return [case["seqlen"]] * case["batch"]
    rng = np.random.Generator(np.random.PCG64(case["lengths_seed"]))
    raw = rng.lognormal(case["len_mu"], case["len_sigma"], case["batch"])
    return [int(x) for x in np.clip(np.rint(raw), case["len_min"], case["len_max"])]


def _is_norm(case):
    return case["kind"] in ("norm", "norm_bwd")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    """Tensors of the case on the GPU, from the seed alone: standard-normal activations, with
    queries and keys of length one, as the rule's layers leave them (rounded to bf16 for bf16
    cases); write strengths sigmoid(x); decays that vary from token to token and from head to
    head, with horizons from tens to thousands of tokens; states of the size that such a past
    leaves; a residual stream a few times as large as what a layer adds, norm weights near one."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(case)

    def randn(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return x.mul_(scale).to(dtype)

    if _is_norm(case):
        rows, width = case["rows"], case["width"]
        t = {"weight": 1.0 + 0.1 * randn(width)}
        if case["kind"] == "norm":
            t["x"] = randn(rows, width, dtype=dt)
            t["residual"] = randn(rows, width, dtype=dt, scale=4.0) if case["residual"] else None
        else:
            t["sum"] = randn(rows, width, dtype=dt, scale=4.0)
            t["dout"], t["dsum"] = randn(rows, width, dtype=dt), randn(rows, width, dtype=dt)
        return t
    H, V, d, B = case["heads"], case["value_heads"], case["head_dim"], case["batch"]
    lengths = _lengths(case)
    t = {"cu": None, "max_seqlen": None}
    if case["layout"] == "ragged":
        t["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32,
                               device="cuda")
        t["max_seqlen"] = max(lengths)

    def act(heads):
        if t["cu"] is not None:
            return (heads, sum(lengths), d)
        return (B, heads, d) if case["kind"] == "delta_step" else (B, heads, case["seqlen"], d)

    def unit(heads):
        x = randn(*act(heads))
        return (x * torch.rsqrt(x.square().sum(-1, keepdim=True))).to(dt)

    t["q"], t["k"], t["v"] = unit(H), unit(H), randn(*act(V), dtype=dt)
    gates = act(V)[:-1]
    rate = torch.exp2(-torch.linspace(3.0, 9.0, V, device="cuda"))
    rate = rate if case["kind"] == "delta_step" else rate[:, None]
    t["log_decay"] = -rate * torch.nn.functional.softplus(2.0 * randn(*gates))
    t["beta"] = torch.sigmoid(randn(*gates))
    t["state"] = None
    if case["kind"] == "delta_step":
        t["state"] = randn(case["slots"], V, d, d)
        t["slots"] = torch.randperm(case["slots"], generator=g, device="cuda")[:B].to(torch.int32)
    elif case["state"]:
        t["state"] = randn(B, V, d, d)
    if case["kind"] == "delta_bwd":
        t["dout"] = randn(*act(V), dtype=dt)
        t["dstate"] = randn(B, V, d, d, scale=0.1) if case["state"] else None
    return t


def prepare(case, seed):
    """The inputs, the batch's chunk table for the plain form, and the scratch that a serving
    loop or a training step keeps from call to call."""
    t = _inputs(case, seed)
    t["case"] = case
    t["table"] = _table(case) if case["kind"] in ("delta", "delta_bwd") else None
    t["workspace"] = None
    return t


def _workspace(t):
    """The scratch that a program keeps for its calls, made at the first of them."""
    from paper_2606_07317_amd import gbla
    if t["workspace"] is None:
        case = t["case"]
        if case["kind"] == "norm_bwd":
            n = gbla.add_rms_norm_backward_workspace_bytes(gbla.norm_shape(t["sum"], EPS))
        else:
            shape = gbla.delta_shape(t["q"], t["k"], t["v"], None, t["cu"], t["max_seqlen"])
            size = gbla.delta_workspace_bytes if case["kind"] == "delta" else gbla.delta_backward_workspace_bytes
            n = size(shape, t["cu"] is not None)
        t["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return t["workspace"]


def run(state):
    t = state
    return _run_own(t) if own else _run_plain(t)


def _run_own(t):
    from paper_2606_07317_amd import gbla
    case = t["case"]
    kind = case["kind"]
    if kind == "norm":
        if not case["bits8"]:
            out, total = gbla.add_rms_norm(t["x"], t["weight"], t["residual"], EPS)
            return {"out": out, "sum": total}
        out, scales, total = gbla.add_rms_norm_e4m3(t["x"], t["weight"], t["residual"], EPS,
                                                    group=case["group"])
        return {"out": _worth(out, scales), "sum": total}
    if kind == "norm_bwd":
        return gbla.add_rms_norm_backward(t["sum"], t["weight"], t["dout"], t["dsum"], EPS,
                                          workspace=_workspace(t))
    if kind == "delta_step":
        out = gbla.delta_step(t["q"], t["k"], t["v"], t["log_decay"], t["beta"], t["state"],
                              state_indices=t["slots"])
        return {"out": out, "state": t["state"]}
    how = dict(initial_state=t["state"], cu_seqlens=t["cu"], max_seqlen=t["max_seqlen"],
               workspace=_workspace(t))
    if kind == "delta":
        out, final = gbla.delta_attention(t["q"], t["k"], t["v"], t["log_decay"], t["beta"],
                                          final_state=True, **how)
        return {"out": out, "final_state": final}
    return gbla.delta_attention_backward(t["q"], t["k"], t["v"], t["log_decay"], t["beta"], t["dout"],
                                         dfinal_state=t["dstate"], **how)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if _is_norm(case):
        rows, width = case["rows"], case["width"]
        n = rows * width
        if kind == "norm_bwd":  # the sum and both gradients once, one gradient out; the weights'
            return {"bytes": 4 * n * e + 8 * width, "flops": 10.0 * n}
        moved = n * e * (3 if case["residual"] else 1)  # x (and the residual, and their sum)
        if case["bits8"]:
            moved += n + 4 * rows * (width // (case["group"] or width))
        else:
            moved += n * e
        return {"bytes": moved + 4 * width, "flops": 6.0 * n}
    H, V, d, B = case["heads"], case["value_heads"], case["head_dim"], case["batch"]
    states = 4.0 * B * V * d * d
    tokens = sum(_lengths(case))
    if kind == "delta_step":
        return {"bytes": 2 * states + B * (2 * H + 2 * V) * d * e + B * (8 * V + 4),
                "flops": 7.0 * B * V * d * d}
    # q, k, v, the gates and the output once, the final state (and the initial one) once; the
    # recurrence's products S^T k, k u^T and S^T q
    cu = 4 * (B + 1) if case["layout"] == "ragged" else 0
    if kind == "delta":
        return {"bytes": tokens * ((2 * H + 2 * V) * d * e + 8 * V) + states * (2 if case["state"] else 1) + cu,
                "flops": tokens * 6.0 * d * d * V}
    # the output's gradient too, and a gradient of each; the states again (S^T k, k u^T), their
    # gradients D (q do^T, D^T k, k dv^T), S do, D u and S dv
    return {"bytes": tokens * ((4 * H + 3 * V) * d * e + 16 * V) + states * (3 if case["state"] else 0) + cu,
            "flops": tokens * 16.0 * d * d * V}


# ---------------------------------------------------------------------------
# The plain forms: elementary torch operations in 32 bits (cumulative decays and long sums
# in 64).
# ---------------------------------------------------------------------------
def _run_plain(t):
    kind = t["case"]["kind"]
    if kind == "norm":
        return _plain_norm(t)
    if kind == "norm_bwd":
        return _plain_norm_bwd(t)
    if kind == "delta_step":
        return _plain_step(t)
    return _plain_delta(t) if kind == "delta" else _plain_delta_bwd(t)


def _worth(out, scales):
    """The values that 8 bits and their scales stand for, in the type of activations."""
    rows, width = out.shape
    y = out.float().view(rows, scales.shape[1], -1) * scales[:, :, None]
    return y.view(rows, width).to(torch.bfloat16)


def _plain_norm(t):
    case = t["case"]
    x = t["x"]
    s = x if t["residual"] is None else (x.float() + t["residual"].float()).to(x.dtype)
    f = s.float()
    y = f * torch.rsqrt((f * f).mean(dim=-1, keepdim=True) + EPS) * t["weight"]
    if not case["bits8"]:
        return {"out": y.to(x.dtype), "sum": s}
    g = y.view(case["rows"], -1, case["group"] or case["width"])
    scales = (g.abs().amax(dim=-1) / 448.0).clamp(min=2.0 ** -126)
    out = (g / scales[:, :, None]).to(torch.float8_e4m3fn).view(y.shape)
    return {"out": _worth(out, scales), "sum": s}


def _plain_norm_bwd(t):
    f, dy = t["sum"].float(), t["dout"].float()
    r = torch.rsqrt((f * f).mean(dim=-1, keepdim=True) + EPS)
    n = f * r
    u = dy * t["weight"]
    dx = t["dsum"].float() + r * (u - n * (u * n).mean(dim=-1, keepdim=True))
    return {"dx": dx.to(t["sum"].dtype), "dweight": (dy * n).sum(dim=0, dtype=torch.float64).float()}


def _plain_step(t):
    case = t["case"]
    V, d = case["value_heads"], case["head_dim"]
    G = V // case["heads"]
    q, k = (t[n].float().repeat_interleave(G, dim=1) for n in ("q", "k"))
    slots = t["slots"].long()
    S = t["state"][slots] * torch.exp(t["log_decay"])[..., None, None]
    u = t["beta"][..., None] * (t["v"].float() - (k[..., :, None] * S).sum(dim=2))
    S = S + k[..., :, None] * u[..., None, :]
    t["state"][slots] = S
    out = (q[..., :, None] * S).sum(dim=2) * d ** -0.5
    return {"out": out.to(t["q"].dtype), "state": t["state"]}


CHUNK = 64


def _table(case):
    """Chunks of at most CHUNK tokens of every sequence: the token that each place of a chunk
    holds (or the one past the last token), each chunk's sequence, and each sequence's first
    and last chunk."""
    seq, size, base, first, last = [], [], [], [], []
    at = 0
    for s, n in enumerate(_lengths(case)):
        first.append(len(seq))
        for c in range(0, n, CHUNK):
            seq.append(s), size.append(min(CHUNK, n - c)), base.append(at + c)
        last.append(len(seq) - 1)
        at += n
    to = lambda x: torch.tensor(x, device="cuda", dtype=torch.int64)
    seq, size, base = to(seq), to(size), to(base)
    i = torch.arange(CHUNK, device="cuda")
    live = i < size[:, None]
    index = torch.where(live, base[:, None] + i, at)
    back = torch.nonzero(live.reshape(-1)).reshape(-1)
    return dict(seq=seq, index=index.reshape(-1), back=back, first=to(first), last=to(last))


def _chunks(x, t, heads):
    """x as [heads, chunks, CHUNK, d] in 32 bits, zeros past the sequences' ends; fewer heads
    than that are repeated."""
    if t["cu"] is None:
        x = x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[-1])
    x = torch.cat([x.float(), torch.zeros_like(x[:, :1], dtype=torch.float32)], dim=1)
    x = x[:, t["table"]["index"]].view(x.shape[0], -1, CHUNK, x.shape[-1])
    return x.repeat_interleave(heads // x.shape[0], dim=0)


def _unchunk(y, like, t):
    """Back to the layout and type of `like`, summed over the heads that share one of its."""
    H = like.shape[0 if t["cu"] is not None else 1]
    y = y.reshape(H, y.shape[0] // H, -1, like.shape[-1]).sum(dim=1)[:, t["table"]["back"]]
    if t["cu"] is None:
        y = y.view(H, like.shape[0], like.shape[2], -1).transpose(0, 1)
    return y.to(like.dtype).contiguous()


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A [.., CHUNK, CHUNK], from blocks of one row to
    the whole: the lower left of two neighbouring blocks X, Y is -Y^-1 A X^-1."""
    T = torch.eye(CHUNK, device=A.device).expand_as(A).contiguous()
    m = 1
    while m < CHUNK:
        n = CHUNK // (2 * m)
        cut = lambda X, r, c: torch.stack([X[..., 2 * m * i + m * r:2 * m * i + m * (r + 1),
                                             2 * m * i + m * c:2 * m * i + m * (c + 1)] for i in range(n)], dim=-3)
        low = -torch.matmul(torch.matmul(cut(T, 1, 1), cut(A, 1, 0)), cut(T, 0, 0))
        for i in range(n):
            T[..., 2 * m * i + m:2 * m * (i + 1), 2 * m * i:2 * m * i + m] = low[..., i, :, :]
        m *= 2
    return T


def _carried(M, B, t, init, reverse):
    """[heads, chunks, d, d]: what enters each chunk where a chunk takes X to M X + B, from
    `init` [sequences, heads, d, d] at each sequence's first chunk (its last, in reverse), by
    doubling; and what leaves each sequence."""
    b = t["table"]
    seq, begin, end = b["seq"], b["first"], b["last"]
    if reverse:
        M, B, seq = M.flip(1), B.flip(1), seq.flip(0)
        begin, end = len(seq) - 1 - b["last"], len(seq) - 1 - b["first"]
    X = B.clone()
    if init is not None:
        X[:, begin] += torch.matmul(M[:, begin], init.transpose(0, 1))
    P, step = M, 1
    longest = int(math.ceil(max(_lengths(t["case"])) / CHUNK))
    while step < longest:
        same = (seq[step:] == seq[:-step])[None, :, None, None]
        X = torch.cat([X[:, :step], X[:, step:] + torch.matmul(P[:, step:], X[:, :-step]) * same], dim=1)
        P = torch.cat([P[:, :step], torch.matmul(P[:, step:], P[:, :-step]) * same], dim=1)
        step *= 2
    into = torch.zeros_like(X)
    into[:, 1:] = X[:, :-1]
    into[:, begin] = 0.0 if init is None else init.transpose(0, 1)
    left = X[:, end].transpose(0, 1).contiguous()
    return into.flip(1) if reverse else into, left


def _pieces(t):
    """What both directions need of the chunks: with c the cumulative log decay,
    u = beta (v - e^c k S - tril(D k k^T) u), D = e^(c_t - c_s); u = Tb v - W S with
    Tb = (I + beta tril(D k k^T))^-1 beta."""
    V = t["case"]["value_heads"]
    p = dict(q=_chunks(t["q"], t, V), k=_chunks(t["k"], t, V), v=_chunks(t["v"], t, V))
    gate = lambda x: _chunks(x[..., None], t, V)[..., 0]
    p["beta"] = gate(t["beta"])[..., None]
    c = torch.cumsum(gate(t["log_decay"]).double(), dim=-1)
    gap = c[..., :, None] - c[..., None, :]
    i = torch.arange(CHUNK, device="cuda")
    at_or_before = i[:, None] >= i[None, :]
    D = torch.exp(torch.where(at_or_before, gap, 0.0)).float() * at_or_before
    p["into"] = torch.exp(c).float()[..., None]
    p["rest"] = torch.exp(c[..., -1:] - c).float()[..., None]
    p["whole"] = torch.exp(c[..., -1]).float()[..., None, None]
    p["D"], p["strict"] = D, D * (i[:, None] > i[None, :])
    p["L"] = torch.matmul(p["k"], p["k"].transpose(-1, -2).contiguous()) * p["strict"]
    p["T"] = _inverse(p["beta"] * p["L"])
    p["W"] = torch.matmul(p["T"], p["beta"] * p["into"] * p["k"])
    p["Tv"] = torch.matmul(p["T"], p["beta"] * p["v"])
    kr = (p["rest"] * p["k"]).transpose(-1, -2).contiguous()
    p["M"] = p["whole"] * torch.eye(p["k"].shape[-1], device="cuda") - torch.matmul(kr, p["W"])
    p["S"], p["final"] = _carried(p["M"], torch.matmul(kr, p["Tv"]), t, t["state"], False)
    p["u"] = p["Tv"] - torch.matmul(p["W"], p["S"])
    p["qk"] = torch.matmul(p["q"], p["k"].transpose(-1, -2).contiguous()) * D
    return p


def _plain_delta(t):
    p = _pieces(t)
    o = p["into"] * torch.matmul(p["q"], p["S"]) + torch.matmul(p["qk"], p["u"])
    return {"out": _unchunk(o * t["case"]["head_dim"] ** -0.5, t["v"], t), "final_state": p["final"]}


def _plain_delta_bwd(t):
    case = t["case"]
    p = _pieces(t)
    T = lambda x: x.transpose(-1, -2).contiguous()
    q, k, S, u, into, rest = p["q"], p["k"], p["S"], p["u"], p["into"], p["rest"]
    do = _chunks(t["dout"], t, case["value_heads"]) * case["head_dim"] ** -0.5
    inner = torch.matmul(T(p["qk"]), do)
    dR = torch.matmul(T(p["T"]), inner)
    rise = torch.matmul(T(into * q), do) - torch.matmul(T(into * k), p["beta"] * dR)
    N, dS0 = _carried(T(p["M"]), rise, t, t["dstate"], True)  # N: the gradient of the state after
    dR = dR + torch.matmul(T(p["T"]), torch.matmul(rest * k, N))
    dv = p["beta"] * dR
    # pairs of the chunk: the output's, and those of the rule itself
    dqk = torch.matmul(do, T(u))
    dkk = -torch.matmul(dv, T(u)) * p["strict"]
    far_q = into * torch.matmul(do, T(S))
    far_k = -into * torch.matmul(dv, T(S))
    to_end = rest * torch.matmul(u, T(N))
    dq = far_q + torch.matmul(dqk * p["D"], k)
    dk = far_k + to_end + torch.matmul(T(dqk * p["D"]), q) + torch.matmul(dkk + T(dkk), k)
    err = p["v"] - into * torch.matmul(k, S) - torch.matmul(p["L"], u)
    dbeta = (err * dR).sum(dim=-1)
    pairs = (p["qk"] * dqk).double() + (torch.matmul(k, T(k)) * dkk).double()
    ends = (k * to_end).sum(dim=-1, dtype=torch.float64)
    dc = (q * far_q + k * far_k).sum(dim=-1, dtype=torch.float64) - ends
    dc = dc + pairs.sum(dim=-1) - pairs.sum(dim=-2)
    last = ends.sum(dim=-1) + (p["whole"] * S * N).sum(dim=(-1, -2), dtype=torch.float64)
    dg = torch.flip(torch.cumsum(torch.flip(dc, (-1,)), dim=-1), (-1,)) + last[..., None]
    gate = lambda x, like: _unchunk(x.float()[..., None], like[..., None], t)[..., 0].contiguous()
    out = {"dq": _unchunk(dq, t["q"], t), "dk": _unchunk(dk, t["k"], t), "dv": _unchunk(dv, t["v"], t),
           "dlog_decay": gate(dg, t["log_decay"]), "dbeta": gate(dbeta, t["beta"])}
    if t["state"] is not None:
        out["dinitial_state"] = dS0
    return out


# ---------------------------------------------------------------------------
# The same results in 64 bits from the definitions: the recurrence token by token and its
# reverse, all sequences side by side.
# ---------------------------------------------------------------------------
def exact(case, seed):
    t = _inputs(case, seed)
    if _is_norm(case):
        return _exact_norm(case, t)
    if case["kind"] == "delta_step":
        return _exact_step(case, t)
    if max(_lengths(case)) > (200000 if case["kind"] == "delta" else 60000):
        return None  # tens of seconds
    return _exact_delta(case, t)


def _e4m3(x):
    """x rounded to e4m3 (three bits of fraction, steps of 2^-9 below 2^-6), half to even."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp(min=-9))
    return torch.round(x / step) * step


def _exact_norm(case, t):
    w = t["weight"].double()
    if case["kind"] == "norm":
        x = t["x"].double()
        s = x if t["residual"] is None else (x + t["residual"].double()).to(_dtype(case)).double()
        y = s / (s.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        if case["bits8"]:
            g = y.view(case["rows"], -1, case["group"] or case["width"])
            scale = g.abs().amax(-1, keepdim=True) / 448.0
            y = (_e4m3(g / scale) * scale).view(y.shape)
        return {"out": y, "sum": s}
    s, dy = t["sum"].double(), t["dout"].double()
    norm = (s.square().mean(-1, keepdim=True) + EPS).sqrt()
    dx = t["dsum"].double() + dy * w / norm - s * (dy * w * s).mean(-1, keepdim=True) / norm ** 3
    return {"dx": dx, "dweight": (dy * s / norm).sum(0)}


def _exact_step(case, t):
    G, d = case["value_heads"] // case["heads"], case["head_dim"]
    S = t["state"].double()
    outs = []
    for n, s in enumerate(t["slots"].tolist()):
        q, k = (t[x][n].double().repeat_interleave(G, dim=0) for x in ("q", "k"))
        Z = S[s] * torch.exp(t["log_decay"][n].double())[:, None, None]
        miss = t["v"][n].double() - (Z * k[:, :, None]).sum(1)
        S[s] = Z + k[:, :, None] * (t["beta"][n].double()[:, None] * miss)[:, None, :]
        outs.append((S[s] * q[:, :, None]).sum(1) * d ** -0.5)
    return {"out": torch.stack(outs), "state": S}


def _exact_delta(case, t):
    H, V, d, B = case["heads"], case["value_heads"], case["head_dim"], case["batch"]
    G, scale, back = V // H, d ** -0.5, case["kind"] == "delta_bwd"
    lengths = _lengths(case)
    order = sorted(range(B), key=lambda s: -lengths[s])  # the longest first: those alive are in front
    alive = [sum(1 for n in lengths if n > i) for i in range(max(lengths))]
    starts = np.concatenate([[0], np.cumsum(lengths)])[:-1][order]
    start = torch.tensor(starts, device="cuda")
    where = torch.tensor(order, device="cuda")

    def flat(x):  # [tokens, heads, ..]
        x = x if t["cu"] is not None else x.transpose(0, 1).reshape(x.shape[1], -1, *x.shape[3:])
        return x.transpose(0, 1).contiguous()

    x = {n: flat(t[n]) for n in ("q", "k", "v", "log_decay", "beta") + (("dout",) if back else ())}
    total = x["q"].shape[0]

    def at(n, i):  # token i of the sequences alive
        y = x[n][start[:alive[i]] + i].double()
        return y.repeat_interleave(G, dim=1) if n in ("q", "k") else y

    def step(S, i):  # (Z, k, miss, state) of token i
        Z = S[:alive[i]] * torch.exp(at("log_decay", i))[..., None, None]
        k = at("k", i)
        miss = at("v", i) - torch.matmul(k[..., None, :], Z)[..., 0, :]
        return Z, k, miss, Z + k[..., :, None] * (at("beta", i)[..., None] * miss)[..., None, :]

    S = torch.zeros(B, V, d, d, device="cuda", dtype=torch.float64)
    if t["state"] is not None:
        S += t["state"][where].double()
    new = lambda heads, *w: torch.zeros(total, heads, *w, device="cuda", dtype=torch.float64)
    out, kept, SEGMENT = new(V, d), [], 128
    for i in range(len(alive)):
        if back and i % SEGMENT == 0:
            kept.append(S[:alive[i]].clone())
        S[:alive[i]] = step(S, i)[3]
        if not back:
            out[start[:alive[i]] + i] = scale * torch.matmul(at("q", i)[..., None, :], S[:alive[i]])[..., 0, :]

    def shaped(y, like):
        y = y.transpose(0, 1)
        if t["cu"] is None:
            y = y.reshape(y.shape[0], like.shape[0], like.shape[2], *y.shape[2:]).transpose(0, 1)
        return y.contiguous()

    if not back:
        return {"out": shaped(out, t["v"]), "final_state": torch.empty_like(S).index_copy_(0, where, S)}
    g = dict(q=new(H, d), k=new(H, d), v=new(V, d), log_decay=new(V), beta=new(V))
    D = torch.zeros_like(S)
    if t["dstate"] is not None:
        D += t["dstate"][where].double()
    fold = lambda y: y.view(y.shape[0], H, G, d).sum(2)
    for c in reversed(range(len(kept))):
        i0, S, past = c * SEGMENT, kept.pop(), []
        for i in range(i0, min(i0 + SEGMENT, len(alive))):
            past.append(step(S, i))
            S = past[-1][3]
        for i in reversed(range(i0, i0 + len(past))):
            Z, k, miss, S = past.pop()
            a, rows = alive[i], start[:alive[i]] + i
            beta, do = at("beta", i)[..., None], scale * at("dout", i)
            now = D[:a] + at("q", i)[..., :, None] * do[..., None, :]
            g["q"][rows] = fold(torch.matmul(S, do[..., None])[..., 0])
            f = torch.matmul(k[..., None, :], now)[..., 0, :]
            dv = beta * f
            g["v"][rows] = dv
            g["beta"][rows] = (f * miss).sum(-1)
            dk = torch.matmul(now, (beta * miss)[..., None]) - torch.matmul(Z, dv[..., None])
            g["k"][rows] = fold(dk[..., 0])
            now = now - k[..., :, None] * dv[..., None, :]
            g["log_decay"][rows] = (now * Z).sum((-1, -2))
            D[:a] = now * torch.exp(at("log_decay", i))[..., None, None]
    res = {"d" + n: shaped(y, t[n]) for n, y in g.items()}
    if t["state"] is not None:
        res["dinitial_state"] = torch.empty_like(D).index_copy_(0, where, D)
    return res
