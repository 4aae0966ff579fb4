"""Performance cases of the decoder operators: what their users run, over the sizes they run it at.

Three operators, in the order a causal decoder calls them:

``gbla.qk_norm_rope``      RMS norm of every head's queries and keys and the rotation by
                           position, and ``gbla.qk_norm_rope_backward``
``gbla.decay_attention``   causal linear attention with one decay per key head, in chunks
                           (prompts, training), and ``gbla.decay_attention_backward``
``gbla.decay_step``        the same attention for one new token of each row of a batch,
                           reading and updating the states

The listed cases take the repository's own workloads (``paper_2606_07317_amd/inputs.py``,
``perf/cases.py``): its heads, head dims, lengths and packed batches.  ``draw`` gives further
cases of the same ranges: every head dim, both data types, shared key heads, odd lengths.

A case is a dict of plain values:
  kind      "rope", "rope_bwd", "decay", "decay_bwd" or "step"
  layout    "dense" (batch x seqlen) or "ragged" (batch sequences whose lengths are
            lognormal(len_mu, len_sigma) within [len_min, len_max])
  heads, kv_heads, head_dim, dtype ("bf16" / "f32")
  rotary_dim, pairs (adjacent channels rotate together), far (positions are given, and far)
  state     an initial state is given and the final one returned (decay, decay_bwd)
  slots     step only: states held, of which the batch's rows name some
  lengths_seed  ragged only: seeds the lengths, so that a case's size (and so its work) does
            not change with the seed of its inputs

With ``own`` false, ``run`` computes the operators from elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 10000.0


def listed():
    return [
        # One new token of four sequences at far positions: a decoder's call between two
        # steps.  Launches and host time are all there is.
        _rope("rope_bf16_decode_b4_h8_d64", "rope", 4, 1, 8, 8, 64, far=True),
        # The queries and keys of one long prompt.
        _rope("rope_bf16_b1_n32768_h8_d64", "rope", 1, 32768, 8, 8, 64),
        # A training batch's gradients of the same.
        _rope("rope_bwd_bf16_b8_n2048_h16_d64", "rope_bwd", 8, 2048, 16, 16, 64),
        # ... of a packed batch in full precision, wide heads, shared key heads, half of the
        # channels rotated.
        _ragged(_rope("rope_bwd_f32_ragged16_h8_kv2_d128", "rope_bwd", 16, 0, 8, 2, 128,
                      dtype="f32", rotary=64, pairs=True), 7.5, 1.0, 16, 32768),
        # A short full-precision prompt with two heads (the size of the workload tiny_f32, and
        # one token past a round length).
        _decay("decay_f32_b1_n257_h2_d32", "decay", 1, 257, 2, 2, 32, dtype="f32"),
        # One long prompt (the throughput workload's size), whose state the single tokens
        # that follow start from.
        _decay("decay_bf16_b1_n32768_h8_d64", "decay", 1, 32768, 8, 8, 64),
        # Packed prompts of very different lengths that go on from earlier states, wide heads,
        # four query heads to a key head.
        _ragged(_decay("decay_bf16_ragged64_h8_kv2_d128", "decay", 64, 0, 8, 2, 128, state=True),
                7.5, 1.0, 16, 32768),
        # A training batch's gradients.
        _decay("decay_bwd_bf16_b8_n2048_h16_d64", "decay_bwd", 8, 2048, 16, 16, 64),
        # ... of a packed batch with wide heads, from states and with gradients of the states.
        _ragged(_decay("decay_bwd_bf16_ragged16_h8_d128", "decay_bwd", 16, 0, 8, 8, 128,
                       state=True), 7.5, 1.0, 16, 32768),
        # One token of one sequence.
        _step("step_bf16_n1_h8_d64", 1, 1, 8, 8, 64),
        # One token of 64 sequences, whose states lie among those of 128.
        _step("step_bf16_n64_h16_d64", 64, 128, 16, 16, 64),
        # A large serving batch with wide heads, four query heads to a key head.
        _step("step_bf16_n256_h16_kv4_d128", 256, 256, 16, 4, 128),
    ]


def draw(rng):
    # The kinds in the shares of the listed cases; sizes uniform in their logarithm, from the
    # smallest listed to no more work than the largest.
    kind = rng.choice(["rope"] * 2 + ["rope_bwd"] * 2 + ["decay"] * 3 + ["decay_bwd"] * 2 + ["step"] * 3)
    d = rng.choice([32, 64, 64, 128])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 16])
    heads = kv * rng.choice([1, 1, 2, 4] if kv <= 4 else [1, 1, 2] if kv == 8 else [1])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if kind == "step":
        # up to the states of the largest listed case
        rows = _log_int(rng, 1, min(512, 2 ** 24 // (kv * d * d)))
        return _unnamed(_step(None, rows, rows + rng.randrange(64), heads, kv, d, dtype))
    # up to the tokens of one long prompt for eight heads of 64
    top = {"rope": 2 ** 25, "rope_bwd": 2 ** 25, "decay": 2 ** 24, "decay_bwd": 2 ** 23}[kind]
    tokens = _log_int(rng, 1 if kind == "rope" else 16, top // (heads * d))
    batch = min(tokens, _log_int(rng, 1, 64))
    if kind in ("rope", "rope_bwd"):
        case = _rope(None, kind, batch, max(1, tokens // batch), heads, kv, d, dtype,
                     rng.choice([d, d, d // 2]), rng.random() < 0.5, rng.random() < 0.3)
    else:
        case = _decay(None, kind, batch, max(1, tokens // batch), heads, kv, d, dtype,
                      rng.random() < 0.5)
    if batch > 1 and rng.random() < 0.5:
        mean, sigma = max(2.0, tokens / batch), rng.choice([0.5, 1.0])
        case = _ragged(case, math.log(mean) - sigma * sigma / 2, sigma, 1,
                       max(16, int(4 * mean)), rng.randrange(1 << 20))
    return _unnamed(case)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _unnamed(case):
    return {n: x for n, x in case.items() if n != "name"}


def _rope(name, kind, batch, seqlen, heads, kv_heads, d, dtype="bf16", rotary=None, pairs=False,
          far=False):
    return dict(name=name, kind=kind, layout="dense", batch=batch, seqlen=seqlen, heads=heads,
                kv_heads=kv_heads, head_dim=d, dtype=dtype, rotary_dim=d if rotary is None else rotary,
                pairs=pairs, far=far)


def _decay(name, kind, batch, seqlen, heads, kv_heads, d, dtype="bf16", state=False):
    return dict(name=name, kind=kind, layout="dense", batch=batch, seqlen=seqlen, heads=heads,
                kv_heads=kv_heads, head_dim=d, dtype=dtype, state=state)


def _step(name, rows, slots, heads, kv_heads, d, dtype="bf16"):
    return dict(name=name, kind="step", layout="dense", batch=rows, seqlen=1, slots=slots,
                heads=heads, kv_heads=kv_heads, head_dim=d, dtype=dtype)


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


def _inputs(case, seed):
    """Tensors of the case on the GPU, from the seed alone: standard-normal activations, as
    projections and norms leave them (rounded to bf16 for bf16 cases); norm weights near one;
    decays whose horizons go from about 30 tokens on the first head to several thousand on
    the last; states of the size that such a past leaves."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def randn(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return x.mul_(scale).to(dtype)

    H, K, d, B = case["heads"], case["kv_heads"], case["head_dim"], case["batch"]
    lengths = _lengths(case)
    t = {"cu": None, "max_seqlen": None}
    if case["layout"] == "ragged":
        t["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32,
                               device="cuda")
        t["max_seqlen"] = max(lengths)

    def act(heads):
        if t["cu"] is not None:
            return (heads, sum(lengths), d)
        return (B, heads, d) if case["kind"] == "step" else (B, heads, case["seqlen"], d)

    t["q"], t["k"] = randn(*act(H), dtype=dt), randn(*act(K), dtype=dt)
    if case["kind"] in ("rope", "rope_bwd"):
        t["q_w"], t["k_w"] = 1.0 + 0.1 * randn(H, d), 1.0 + 0.1 * randn(K, d)
        t["positions"] = None
        if case["far"]:
            rows = (sum(lengths),) if t["cu"] is not None else (B, case["seqlen"])
            t["positions"] = torch.randint(0, 1 << 20, rows, generator=g, device="cuda",
                                           dtype=torch.int32)
        if case["kind"] == "rope_bwd":
            t["dq_out"], t["dk_out"] = randn(*act(H), dtype=dt), randn(*act(K), dtype=dt)
        return t
    t["v"] = randn(*act(K), dtype=dt)
    horizon = torch.linspace(5.0, 12.0, K, device="cuda") + 0.1 * randn(K)
    t["log_decay"] = torch.log1p(-torch.exp2(-horizon))
    t["state"] = None
    if case["kind"] == "step":
        t["state"] = randn(case["slots"], K, d, d, scale=4.0)
        t["slots"] = torch.randperm(case["slots"], generator=g, device="cuda")[:B].to(torch.int32)
    elif case["state"]:
        t["state"] = randn(B, K, d, d, scale=4.0)
    if case["kind"] == "decay_bwd":
        t["dout"] = randn(*act(H), dtype=dt)
        t["dstate"] = randn(B, K, d, d, scale=0.1) if case["state"] else None
    return t


def prepare(case, seed):
    """The inputs, the batch's chunk table for the plain form, and the scratch and output
    buffers that a serving loop or a training step keeps from call to call."""
    t = _inputs(case, seed)
    t["case"] = case
    t["table"] = _table(case) if case["kind"] in ("decay", "decay_bwd") else None
    t["workspace"] = None
    return t


def _workspace(t):
    """The scratch that a program keeps for its calls, made at the first of them."""
    from paper_2606_07317_amd import gbla
    if t["workspace"] is None:
        kind = t["case"]["kind"]
        if kind == "rope_bwd":
            n = gbla.qk_norm_rope_backward_workspace_bytes(
                gbla.rope_shape(t["q"], t["k"], t["cu"], t["case"]["rotary_dim"], THETA, EPS))
        else:
            shape = gbla.decay_shape(t["q"], t["k"], None, t["cu"], t["max_seqlen"])
            n = (gbla.decay_workspace_bytes(shape) if kind == "decay"
                 else gbla.decay_backward_workspace_bytes(shape))
        t["workspace"] = torch.empty(n, dtype=torch.uint8, device=t["q"].device)
    return t["workspace"]


def run(state):
    t = state
    return _run_own(t) if own else _run_plain(t)


def _run_own(t):
    from paper_2606_07317_amd import gbla
    case = t["case"]
    kind = case["kind"]
    if kind == "step":
        out = gbla.decay_step(t["q"], t["k"], t["v"], t["log_decay"], t["state"],
                              state_indices=t["slots"])
        return {"out": out, "state": t["state"]}
    if kind == "decay":
        out, final = gbla.decay_attention(t["q"], t["k"], t["v"], t["log_decay"],
                                          initial_state=t["state"], final_state=True,
                                          cu_seqlens=t["cu"], max_seqlen=t["max_seqlen"],
                                          workspace=_workspace(t))
        return {"out": out, "final_state": final}
    if kind == "decay_bwd":
        return gbla.decay_attention_backward(t["q"], t["k"], t["v"], t["log_decay"], t["dout"],
                                             initial_state=t["state"], dfinal_state=t["dstate"],
                                             cu_seqlens=t["cu"], max_seqlen=t["max_seqlen"],
                                             workspace=_workspace(t))
    flags = gbla.ROPE_PAIRS if case["pairs"] else 0
    how = dict(positions=t["positions"], cu_seqlens=t["cu"], rotary_dim=case["rotary_dim"],
               theta=THETA, eps=EPS, flags=flags)
    if kind == "rope":
        q, k = gbla.qk_norm_rope(t["q"], t["k"], t["q_w"], t["k_w"], **how)
        return {"q": q, "k": k}
    return gbla.qk_norm_rope_backward(t["q"], t["k"], t["q_w"], t["k_w"], t["dq_out"], t["dk_out"],
                                      workspace=_workspace(t), **how)


def work(case):
    H, K, d, B = case["heads"], case["kv_heads"], case["head_dim"], case["batch"]
    tokens = sum(_lengths(case))
    e = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    cu = 4 * (B + 1) if case["layout"] == "ragged" else 0
    if kind in ("rope", "rope_bwd"):
        # q and k once, the rotated ones once; backward: the cotangents too
        rows = tokens * (H + K) * d
        extra = cu + 4 * (H + K) * d * (2 if kind == "rope_bwd" else 1)
        extra += 4 * tokens if case["far"] else 0
        return {"bytes": rows * e * (3 if kind == "rope_bwd" else 2) + extra,
                "flops": rows * (16.0 if kind == "rope_bwd" else 8.0)}
    states = 4.0 * B * K * d * d
    if kind == "step":
        return {"bytes": 2 * states + B * (2 * H + 2 * K) * d * e + 4 * B + 4 * K,
                "flops": 3.0 * B * K * d * d + 2.0 * B * H * d * d}
    # q, k, v and the output once, the final state (and the initial one) once; the recurrence's
    # products: k v^T a key head, S^T q a query head
    if kind == "decay":
        return {"bytes": tokens * (2 * H + 2 * K) * d * e + states * (2 if case["state"] else 1) + cu + 4 * K,
                "flops": tokens * 2.0 * d * d * (K + H)}
    # the output's gradient too, and a gradient of each; both states' products, S do, D v, D^T k
    return {"bytes": tokens * (3 * H + 4 * K) * d * e + states * (3 if case["state"] else 0) + cu + 8 * K,
            "flops": tokens * 2.0 * d * d * (2 * H + 3 * K)}


# ---------------------------------------------------------------------------
# The plain forms: elementary torch operations in 32 bits (angles in 64).
# ---------------------------------------------------------------------------
def _run_plain(t):
    kind = t["case"]["kind"]
    if kind == "step":
        return _plain_step(t)
    if kind == "decay":
        return _plain_decay(t)
    if kind == "decay_bwd":
        return _plain_decay_bwd(t)
    return _plain_rope(t) if kind == "rope" else _plain_rope_bwd(t)


def _positions(t):
    """Positions [B, 1, n] or [1, T]: given, or counted from each sequence's start."""
    q = t["q"]
    if t["positions"] is not None:
        return t["positions"].unsqueeze(-2)
    if t["cu"] is None:
        return torch.arange(q.shape[-2], device=q.device).view(1, 1, -1)
    at = torch.arange(q.shape[-2], device=q.device)
    start = t["cu"][torch.searchsorted(t["cu"], at.to(torch.int32), right=True) - 1]
    return (at - start).view(1, -1)


def _angles(t):
    R = t["case"]["rotary_dim"]
    inv = torch.pow(THETA, -torch.arange(0, R, 2, device=t["q"].device, dtype=torch.float64) / R)
    a = _positions(t).double()[..., None] * inv
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(x, cos, sin, R, pairs):
    y = x.clone()
    if pairs:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_rope(t):
    case = t["case"]
    cos, sin = _angles(t)

    def one(x, w):
        f = x.float()
        f = f * torch.rsqrt((f * f).mean(dim=-1, keepdim=True) + EPS) * w[:, None, :]
        return _rotate(f, cos, sin, case["rotary_dim"], case["pairs"]).to(x.dtype)

    return {"q": one(t["q"], t["q_w"]), "k": one(t["k"], t["k_w"])}


def _plain_rope_bwd(t):
    case = t["case"]
    cos, sin = _angles(t)

    def one(x, w, dy):
        f = x.float()
        r = torch.rsqrt((f * f).mean(dim=-1, keepdim=True) + EPS)
        n = f * r
        u = _rotate(dy.float(), cos, -sin, case["rotary_dim"], case["pairs"])
        dw = u * n
        dw = dw.sum(dim=(0, 2)) if dw.dim() == 4 else dw.sum(dim=1)
        u = u * w[:, None, :]
        return (r * (u - n * (u * n).mean(dim=-1, keepdim=True))).to(x.dtype), dw

    dq, dq_w = one(t["q"], t["q_w"], t["dq_out"])
    dk, dk_w = one(t["k"], t["k_w"], t["dk_out"])
    return {"dq": dq, "dk": dk, "dq_w": dq_w, "dk_w": dk_w}


def _plain_step(t):
    case = t["case"]
    N, K, d = case["batch"], case["kv_heads"], case["head_dim"]
    q = t["q"].float().view(N, K, -1, d)
    slots = t["slots"].long()
    lam = torch.exp(t["log_decay"]).view(1, K, 1, 1)
    S = t["state"][slots] * lam + t["k"].float()[..., :, None] * t["v"].float()[..., None, :]
    t["state"][slots] = S
    out = torch.matmul(q, S) * d ** -0.5
    return {"out": out.view(N, -1, d).to(t["q"].dtype), "state": t["state"]}


CHUNK = 128


def _table(case):
    """Chunks of at most CHUNK tokens of every sequence: the token that each place of a chunk
    holds (or the one past the last token), and each chunk's sequence, start, length and its
    sequence's length."""
    seq, start, size, total, base = [], [], [], [], []
    at = 0
    for s, n in enumerate(_lengths(case)):
        for c in range(0, n, CHUNK):
            seq.append(s), start.append(c), size.append(min(CHUNK, n - c)), total.append(n)
            base.append(at + c)
        at += n
    to = lambda x: torch.tensor(x, device="cuda", dtype=torch.int64)
    seq, start, size, total, base = to(seq), to(start), to(size), to(total), to(base)
    i = torch.arange(CHUNK, device="cuda")
    live = i < size[:, None]
    index = torch.where(live, base[:, None] + i, at)
    back = torch.nonzero(live.reshape(-1)).reshape(-1)
    return dict(seq=seq, start=start, size=size, total=total, index=index, back=back)


def _chunks(x, t, group):
    """x as [K, group, chunks, CHUNK, d] in 32 bits, zeros past the sequences' ends."""
    if x.dim() == 4:
        x = x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])
    x = torch.cat([x.float(), torch.zeros_like(x[:, :1], dtype=torch.float32)], dim=1)
    x = x[:, t["table"]["index"].reshape(-1)]
    return x.view(-1, group, t["table"]["index"].shape[0], CHUNK, x.shape[-1])


def _unchunk(y, like, t):
    y = y.reshape(like.shape[-3], -1, like.shape[-1])[:, t["table"]["back"]]
    if like.dim() == 4:
        y = y.view(like.shape[1], like.shape[0], like.shape[2], -1).transpose(0, 1)
    return y.to(like.dtype).contiguous()


def _decays(t):
    """The decay's powers (in 64 bits, rounded to 32) that the chunks need, a key head first:
    within a chunk, from its start to a token, from a token to its end, over a whole one,
    from chunk to chunk of a sequence, from a sequence's start, to its end."""
    b = t["table"]
    g = t["log_decay"].double()
    power = lambda e: torch.exp(g.view(-1, *[1] * e.dim()) * e).float()
    i = torch.arange(CHUNK, device="cuda").double()
    gap = (i[:, None] - i[None, :])
    end = b["start"] + b["size"]
    to_end = (b["size"][:, None] - 1 - i).clamp(min=0)
    follows = (b["seq"][:, None] == b["seq"][None, :]) & (b["start"][:, None] > b["start"][None, :])
    between = torch.where(follows, b["start"][:, None] - end[None, :], 0).double()
    return dict(
        gap=gap.clamp(min=0).float(), inside=power(gap.clamp(min=0)) * (gap >= 0),
        into=power(i + 1), to_end=power(to_end), left=to_end.float(), whole=power(b["size"].double()),
        between=power(between) * follows, before=power(b["start"].double()),
        after=power((b["total"] - end).double()))


def _entering(part, p):
    """[K, chunks, d, d] parts carried into each later chunk of their sequence."""
    K, C, d, _ = part.shape
    return torch.bmm(p["between"], part.reshape(K, C, d * d)).view(K, C, d, d)


def _leaving(part, p):
    K, C, d, _ = part.shape
    back = p["between"].transpose(1, 2).contiguous()
    return torch.bmm(back, part.reshape(K, C, d * d)).view(K, C, d, d)


def _by_sequence(x, weight, t):
    """sum over the chunks of a sequence of weight * x: [sequences, K, d, d]."""
    out = torch.zeros((t["case"]["batch"],) + (x.shape[0],) + x.shape[2:], device=x.device)
    return out.index_add_(0, t["table"]["seq"], (x * weight[..., None, None]).transpose(0, 1))


def _whole(t, K):
    """The decay over each whole sequence [sequences, K, 1, 1]."""
    n = torch.tensor(_lengths(t["case"]), device="cuda").double()
    return torch.exp(n[:, None] * t["log_decay"].double()).float()[..., None, None]


def _states(t, k, v, p):
    """Each chunk's own k v^T, and the state before each chunk."""
    part = torch.matmul((k * p["to_end"][:, :, :, None]).transpose(-1, -2), v)
    S = _entering(part, p)
    if t["state"] is not None:
        S = S + t["state"][t["table"]["seq"]].transpose(0, 1) * p["before"][..., None, None]
    return part, S


def _plain_decay(t):
    case = t["case"]
    K, G = case["kv_heads"], case["heads"] // case["kv_heads"]
    scale = case["head_dim"] ** -0.5
    p = _decays(t)
    q = _chunks(t["q"], t, G)
    k, v = _chunks(t["k"], t, 1)[:, 0], _chunks(t["v"], t, 1)[:, 0]
    part, S = _states(t, k, v, p)
    o = torch.matmul(q, S[:, None]) * p["into"][:, None, None, :, None]
    w = torch.matmul(q, k.transpose(-1, -2)[:, None]) * p["inside"][:, None, None]
    o = (o + torch.matmul(w, v[:, None])) * scale
    final = _by_sequence(part, p["after"], t)
    if t["state"] is not None:
        final = final + t["state"] * _whole(t, K)
    return {"out": _unchunk(o, t["q"], t), "final_state": final}


def _plain_decay_bwd(t):
    case = t["case"]
    K, G = case["kv_heads"], case["heads"] // case["kv_heads"]
    scale = case["head_dim"] ** -0.5
    b, p = t["table"], _decays(t)
    q, do = _chunks(t["q"], t, G), _chunks(t["dout"], t, G) * scale
    k, v = _chunks(t["k"], t, 1)[:, 0], _chunks(t["v"], t, 1)[:, 0]
    part, S = _states(t, k, v, p)
    # the gradient of the state after each chunk
    rise = (torch.matmul((q * p["into"][:, None, None, :, None]).transpose(-1, -2), do)).sum(dim=1)
    D = _leaving(rise, p)
    if t["dstate"] is not None:
        D = D + t["dstate"][b["seq"]].transpose(0, 1) * p["after"][..., None, None]
    qk = torch.matmul(q, k.transpose(-1, -2)[:, None]) * p["inside"][:, None, None]
    dov = torch.matmul(do, v.transpose(-1, -2)[:, None])
    inner = (qk * dov * p["gap"]).sum(dim=(1, 2, 3, 4))
    dov = dov * p["inside"][:, None, None]
    far_q = torch.matmul(do, S.transpose(-1, -2)[:, None]) * p["into"][:, None, None, :, None]
    dq = far_q + torch.matmul(dov, k[:, None])
    far_k = torch.matmul(v, D.transpose(-1, -2)) * p["to_end"][..., None]
    dk = far_k + torch.matmul(dov.transpose(-1, -2), q).sum(dim=1)
    dv = torch.matmul(k, D) * p["to_end"][..., None] + torch.matmul(qk.transpose(-1, -2), do).sum(dim=1)
    i = torch.arange(1, CHUNK + 1, device="cuda", dtype=torch.float32)
    dg = inner + ((q * far_q).sum(dim=(1, 4)) * i).sum(dim=(1, 2))
    dg = dg + ((k * far_k).sum(dim=3) * p["left"]).sum(dim=(1, 2))
    dg = dg + ((S * D).sum(dim=(2, 3)) * p["whole"] * b["size"]).sum(dim=1)
    out = {"dq": _unchunk(dq, t["q"], t), "dk": _unchunk(dk, t["k"], t), "dv": _unchunk(dv, t["v"], t),
           "dlog_decay": dg}
    if t["state"] is not None:
        out["dinitial_state"] = _by_sequence(rise, p["before"], t) + t["dstate"] * _whole(t, K)
    return out


# ---------------------------------------------------------------------------
# The same results in 64 bits from the definitions: sums over all earlier tokens, a block of
# rows at a time; rotations as products of complex numbers.
# ---------------------------------------------------------------------------
def exact(case, seed):
    t = _inputs(case, seed)
    t["case"] = case
    if case["kind"] in ("rope", "rope_bwd"):
        return _exact_rope(case, t)
    if case["kind"] == "step":
        return _exact_step(case, t)
    pairs = sum(n * n for n in _lengths(case)) * case["heads"]
    if pairs * (2 if case["kind"] == "decay" else 5) * case["head_dim"] > 8e13:
        return None  # tens of seconds
    return _exact_decay(case, t)


def _exact_rope(case, t):
    R, d = case["rotary_dim"], case["head_dim"]
    where = []
    if t["positions"] is not None:
        where = t["positions"].double()
    elif t["cu"] is None:
        where = torch.arange(case["seqlen"], device="cuda").double().expand(case["batch"], -1)
    else:
        where = torch.cat([torch.arange(n, device="cuda").double() for n in _lengths(case)])
    freq = torch.tensor([THETA ** (-2.0 * i / R) for i in range(R // 2)], device="cuda",
                        dtype=torch.float64)
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), where[..., None] * freq)
    turn = turn.unsqueeze(-3)
    if case["pairs"]:
        order = list(range(d))
    else:
        order = [c for i in range(R // 2) for c in (i, i + R // 2)] + list(range(R, d))
    order = torch.tensor(order, device="cuda")

    def spin(x, by):
        x = x[..., order]
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous())
        x = torch.cat([torch.view_as_real(z * by).flatten(-2), x[..., R:]], dim=-1)
        return torch.empty_like(x).index_copy_(-1, order, x)

    out = {}
    for n in ("q", "k"):
        x, w = t[n].double(), t[n + "_w"].double()[:, None, :]
        norm = x.square().mean(-1, keepdim=True).add(EPS).sqrt()
        if case["kind"] == "rope":
            out[n] = spin(x / norm * w, turn)
            continue
        u = spin(t["d" + n + "_out"].double(), turn.conj())
        dims = [i for i in range(x.dim()) if i not in (x.dim() - 3, x.dim() - 1)]
        out["d" + n + "_w"] = (u * x / norm).sum(dims)
        out["d" + n] = u * w / norm - x * (u * w * x).mean(-1, keepdim=True) / norm ** 3
    return out


def _exact_step(case, t):
    K, d = case["kv_heads"], case["head_dim"]
    S = t["state"].double()
    q, k, v = t["q"].double(), t["k"].double(), t["v"].double()
    outs = []
    rows = t["slots"].tolist()
    lam = torch.exp(t["log_decay"].double())[:, None, None]
    for n, s in enumerate(rows):
        S[s] = S[s] * lam + k[n][:, :, None] * v[n][:, None, :]
        wide = S[s].repeat_interleave(case["heads"] // K, dim=0)
        outs.append((q[n][:, :, None] * wide).sum(dim=1) * d ** -0.5)
    return {"out": torch.stack(outs), "state": S}


def _exact_decay(case, t):
    K, G, d, B = case["kv_heads"], case["heads"] // case["kv_heads"], case["head_dim"], case["batch"]
    scale, g = d ** -0.5, t["log_decay"].double()
    back = case["kind"] == "decay_bwd"
    names = ("q", "k", "v") + (("dout",) if back else ())
    grads = {n: torch.zeros(t[n].shape, device="cuda", dtype=torch.float64) for n in names[:3]}
    out = torch.zeros(t["q"].shape, device="cuda", dtype=torch.float64)
    final = torch.zeros((B, K, d, d), device="cuda", dtype=torch.float64)
    dstate = torch.zeros_like(final)
    dg = torch.zeros(K, device="cuda", dtype=torch.float64)
    at = 0
    for s, n in enumerate(_lengths(case)):
        piece = (lambda x: x[s]) if t["cu"] is None else (lambda x: x[:, at:at + n])
        i = torch.arange(n, device="cuda").double()
        for h in range(K):
            k, v = piece(t["k"])[h].double(), piece(t["v"])[h].double()
            S0 = t["state"][s, h].double() if t["state"] is not None else None
            late = torch.exp(g[h] * (n - 1 - i))[:, None]
            early = torch.exp(g[h] * (i + 1))[:, None]
            final[s, h] = (late * k).t() @ v
            if S0 is not None:
                final[s, h] += torch.exp(g[h] * n) * S0
            D = t["dstate"][s, h].double() if back and t["dstate"] is not None else None
            if D is not None:  # the final state's own terms
                piece(grads["k"])[h] += late * (v @ D.t())
                piece(grads["v"])[h] += late * (k @ D)
                dg[h] += ((n - 1 - i)[:, None] * late * k * (v @ D.t())).sum()
                dstate[s, h] += torch.exp(g[h] * n) * D
                if S0 is not None:
                    dg[h] += n * torch.exp(g[h] * n) * (S0 * D).sum()
            for j in range(h * G, (h + 1) * G):
                q = piece(t["q"])[j].double()
                do = piece(t["dout"])[j].double() * scale if back else None
                for a in range(0, n, 2048):
                    b = min(n, a + 2048)
                    dist = i[a:b, None] - i[None, :b]
                    lam = torch.exp(g[h] * dist.clamp(min=0)) * (dist >= 0)
                    A = (q[a:b] @ k[:b].t()) * lam
                    if not back:
                        y = A @ v[:b]
                        if S0 is not None:
                            y = y + early[a:b] * (q[a:b] @ S0)
                        piece(out)[j][a:b] = scale * y
                        continue
                    dA = (do[a:b] @ v[:b].t()) * lam
                    piece(grads["q"])[j][a:b] += dA @ k[:b]
                    piece(grads["k"])[h][:b] += dA.t() @ q[a:b]
                    piece(grads["v"])[h][:b] += A.t() @ do[a:b]
                    dg[h] += (A * (do[a:b] @ v[:b].t()) * dist).sum()
                    if S0 is not None:
                        far = early[a:b] * (do[a:b] @ S0.t())
                        piece(grads["q"])[j][a:b] += far
                        dg[h] += ((i[a:b] + 1)[:, None] * far * q[a:b]).sum()
                    dstate[s, h] += (early[a:b] * q[a:b]).t() @ do[a:b]
        at += n
    if not back:
        return {"out": out, "final_state": final}
    res = {"dq": grads["q"], "dk": grads["k"], "dv": grads["v"], "dlog_decay": dg}
    if t["state"] is not None:
        res["dinitial_state"] = dstate
    return res
