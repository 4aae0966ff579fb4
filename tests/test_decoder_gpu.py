"""The decoder's operators on the GPU against the 64-bit references.

Tolerances are bounds, not fits.  With u = 2^-24 (half a step of fp32), ``size`` the same
sum with every term's absolute value, and half a step of the result's type for its last
rounding:

* norm and rotation: an entry is a sum of two products, each after at most d / 8 + 24
  roundings (the row's sum of squares, the square root, the quotient, weight, sine or
  cosine with its angle's error of 3 u): (d / 8 + 24) 2 u size.  A matrix unit or a fused
  sum may truncate where an addition rounds, hence the 2.  The weights' gradients add
  sums over the tokens: 32 additions in a lane and 64 over lanes, waves and workgroups
  (compensated): 128 2 u size.
* decay attention: an output's terms pass at most d (scores) + 64 (a tile's sum) + d (the
  state's read) + 64 (a tile's update) additions, one more for every tile and unit that
  the state is carried over and 16 other roundings:  c = (2 d + 144 + n / 64) 2 u size.
  In bf16 the kernels round scores and states to two parts, 2^-17 of a term each:
  c + 2^-16 size.
* the decay's gradient: the same, where ``size`` counts each pair with its distance and
  with 512 (the longest unit, whose passing pairs are a difference).
"""
import pytest
import torch

from oracle import gbla_decoder as ref
from paper_2606_07317_amd import gbla

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(gen, *shape, dtype=F32, scale=1.0):
    return (scale * torch.randn(*shape, generator=gen)).to(dtype)


def _check(got, want, size, c, name):
    """Every entry within half a step of its type and c * size."""
    assert got.shape == want.shape, name
    step = torch.finfo(got.dtype).eps / 2
    got = got.cpu().double()
    assert torch.isfinite(got).all(), name
    over = (got - want).abs() - (step * want.abs() * (1 + 2 * step) + c * size + 1e-37)
    assert (over <= 0).all(), "%s: over its bound by %.3g (of |want| %.3g, size %.3g)" % (
        name, over.max(), want.reshape(-1)[over.argmax()].abs(), size.reshape(-1)[over.argmax()])


def _dev(*ts):
    return [None if t is None else t.cuda() for t in ts]


# ---------------------------------------------------------------------------
# Norm and rotation
# ---------------------------------------------------------------------------
ROPE = [
    # lengths, ragged, H, K, d, rotary, flags, dtype, positions given
    ([1], False, 1, 1, 32, 32, 0, F32, True),
    ([1] * 5, False, 8, 8, 64, 64, 0, BF16, True),
    ([300] * 2, False, 3, 3, 64, 64, 0, BF16, False),
    ([131] * 3, False, 8, 2, 128, 64, gbla.ROPE_PAIRS, F32, False),
    ([77], False, 2, 5, 32, 8, gbla.ROPE_PAIRS, BF16, False),
    ([65] * 2, False, 4, 2, 128, 128, 0, BF16, True),
    ([100], False, 2, 1, 64, 0, 0, F32, False),
    ([100], False, 2, 1, 64, 32, gbla.NO_NORM, F32, False),
    ([3, 0, 129, 1, 40], True, 4, 1, 64, 64, 0, F32, False),
    ([3, 0, 129, 1, 40], True, 2, 2, 128, 96, gbla.ROPE_PAIRS | gbla.NO_NORM, BF16, False),
    ([0, 0, 17], True, 12, 4, 32, 16, 0, BF16, True),
]


def _rope_case(lengths, ragged, H, K, d, rotary, flags, dtype, given, seed=0):
    gen = _gen(seed)
    T, B, n = sum(lengths), len(lengths), lengths[0]
    act = (lambda h: (h, T, d)) if ragged else (lambda h: (B, h, n, d))
    t = dict(q=_randn(gen, *act(H), dtype=dtype), k=_randn(gen, *act(K), dtype=dtype, scale=3.0),
             dq=_randn(gen, *act(H), dtype=dtype), dk=_randn(gen, *act(K), dtype=dtype),
             q_w=1 + 0.3 * _randn(gen, H, d), k_w=1 + 0.3 * _randn(gen, K, d), pos=None, cu=None)
    if given:
        t["pos"] = torch.randint(0, 2 ** 30, (T,) if ragged else (B, n), generator=gen).to(torch.int32)
    if ragged:
        t["cu"] = torch.tensor([0] + lengths).cumsum(0).to(torch.int32)
    if flags & gbla.NO_NORM:
        t["q_w"] = t["k_w"] = None
    return t


def _each(t, x, lengths, ragged):
    """The batch's sequences of x: views [heads, n, d], and their positions."""
    at = 0
    for s, n in enumerate(lengths):
        if ragged:
            pos = t["pos"][at:at + n] if t["pos"] is not None else torch.arange(n)
            yield x[:, at:at + n], pos
        else:
            yield x[s], t["pos"][s] if t["pos"] is not None else torch.arange(n)
        at += n


def _pair_size(x, rotary, adjacent):
    """|a| + |b| in both channels of a pair."""
    y = x.abs()
    if rotary:
        a, b = ref._pairs(x.shape[-1], rotary, adjacent)
        y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(map(str, c[1:8])))
def test_rope(case):
    lengths, ragged, H, K, d, rotary, flags, dtype, _ = case
    t = _rope_case(*case)
    adjacent = bool(flags & gbla.ROPE_PAIRS)
    how = dict(positions=t["pos"], cu_seqlens=t["cu"])
    got = gbla.qk_norm_rope(*_dev(t["q"], t["k"], t["q_w"], t["k_w"]), rotary_dim=rotary, flags=flags,
                            **{n: _dev(x)[0] for n, x in how.items()})
    for name, x, w, y in (("q", t["q"], t["q_w"], got[0]), ("k", t["k"], t["k_w"], got[1])):
        assert y.dtype == dtype
        for (xs, pos), (ys, _) in zip(_each(t, x, lengths, ragged), _each(t, y, lengths, ragged)):
            want = ref.rope(xs, w, pos, rotary, adjacent=adjacent)
            size = _pair_size(ref.rope(xs, w, pos, 0), rotary, adjacent)
            _check(ys, want, size, (d / 8 + 24) * 2 * U, name)


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(map(str, c[1:8])))
def test_rope_backward(case):
    lengths, ragged, H, K, d, rotary, flags, dtype, _ = case
    t = _rope_case(*case)
    adjacent = bool(flags & gbla.ROPE_PAIRS)
    how = {n: _dev(x)[0] for n, x in dict(positions=t["pos"], cu_seqlens=t["cu"]).items()}
    g = gbla.qk_norm_rope_backward(*_dev(t["q"], t["k"], t["q_w"], t["k_w"], t["dq"], t["dk"]),
                                   rotary_dim=rotary, flags=flags, **how)
    for n in ("q", "k"):
        x, w, dy = t[n], t[n + "_w"], t["d" + n]
        dw, dw_size = 0.0, 0.0
        for (xs, pos), (dys, _), (gs, _) in zip(*(_each(t, z, lengths, ragged)
                                                  for z in (x, dy, g["d" + n]))):
            want, part = ref.rope_backward(xs, w, pos, dys, rotary, adjacent=adjacent)
            u = _pair_size(dys.double(), rotary, adjacent)
            if w is not None:
                r = 1 / torch.sqrt((xs.double() ** 2).mean(-1, keepdim=True) + 1e-6)
                xn, uw = (xs.double() * r).abs(), u * w.double()[:, None, :].abs()
                dw, dw_size = dw + part, dw_size + (u * xn).sum(1)
                u = r * (uw + xn * (uw * xn).mean(-1, keepdim=True))
            _check(gs, want, u, (d / 8 + 40) * 2 * U, "d" + n)
        if w is None:
            assert "d%s_w" % n not in g
        else:
            _check(g["d%s_w" % n], dw, dw_size, 192 * 2 * U, "d%s_w" % n)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rope_in_place_and_into_given_outputs(dtype):
    t = _rope_case([200] * 2, False, 4, 2, 64, 64, 0, dtype, True)
    q, k, q_w, k_w, pos, dq, dk = _dev(*(t[n] for n in ("q", "k", "q_w", "k_w", "pos", "dq", "dk")))
    want = gbla.qk_norm_rope(q, k, q_w, k_w, positions=pos)
    wg = gbla.qk_norm_rope_backward(q, k, q_w, k_w, dq, dk, positions=pos)
    gg = gbla.qk_norm_rope_backward(q, k, q_w, k_w, dq, dk, positions=pos, grads=dict(dq=dq, dk=dk))
    assert gg["dq"] is dq and torch.equal(dq, wg["dq"]) and torch.equal(dk, wg["dk"])
    got = gbla.qk_norm_rope(q, k, q_w, k_w, positions=pos, q_out=q, k_out=k)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rope_weight_gradients_over_many_tokens():
    """More tokens than one pass of a workgroup takes, and repeated calls give the same bits."""
    gen = _gen(3)
    n, H, d = 70001, 16, 32
    q, dy = _randn(gen, 1, H, n, d, dtype=BF16), _randn(gen, 1, H, n, d, dtype=BF16)
    w = 1 + 0.3 * _randn(gen, H, d)
    args = _dev(q, q, w, w, dy, dy)
    a, b = (gbla.qk_norm_rope_backward(*args) for _ in range(2))
    assert all(torch.equal(a[x], b[x]) for x in a)
    assert torch.equal(a["dq_w"], a["dk_w"]) and torch.equal(a["dq"], a["dk"])
    _, want = ref.rope_backward(q[0], w, torch.arange(n), dy[0], d)
    r = 1 / torch.sqrt((q[0].double() ** 2).mean(-1, keepdim=True) + 1e-6)
    size = (_pair_size(dy[0].double(), d, False) * (q[0].double() * r).abs()).sum(1)
    _check(a["dq_w"], want, size, 192 * 2 * U, "dq_w")


# ---------------------------------------------------------------------------
# Decay attention
# ---------------------------------------------------------------------------
DECAY = [
    # lengths, ragged, H, K, d, dtype, states, log decays of the key heads
    ([1], False, 1, 1, 32, F32, False, [-0.1]),
    ([63] * 2, False, 2, 2, 64, BF16, True, [-0.05, -3.0]),
    ([64], False, 4, 2, 128, BF16, False, [-0.01, 0.0]),
    ([65], False, 4, 1, 128, F32, True, [-0.02]),
    ([200] * 3, False, 6, 2, 32, BF16, True, [-0.001, -30.0]),
    ([257], False, 2, 2, 32, F32, False, [-0.03, -0.0005]),
    ([600], False, 2, 2, 64, BF16, True, [-0.01, -float("inf")]),   # split into units
    ([777] * 2, False, 4, 2, 64, F32, True, [-0.004, -0.3]),
    ([513], False, 3, 1, 128, BF16, True, [-0.008]),
    ([640], False, 2, 2, 128, F32, False, [-0.02, -0.001]),
    ([1300], False, 2, 1, 32, BF16, False, [-0.002]),
    ([5, 0, 130, 1, 64, 300], True, 4, 2, 64, F32, True, [-0.05, -0.002]),
    ([700, 0, 1, 128, 513], True, 2, 1, 64, BF16, True, [-0.01]),
    ([0, 900, 64, 0], True, 2, 2, 128, BF16, False, [-0.01, -1.0]),
    ([33] * 40, True, 8, 8, 32, BF16, False, [-0.01 * (i + 1) for i in range(8)]),
    ([64, 66] * 20, True, 2, 2, 32, F32, True, [-0.1, -0.01]),
]
_IDS = ["%s-%s" % ("ragged" if c[1] else "dense", "-".join(map(str, (len(c[0]), max(c[0])) + c[2:7]))) for c in DECAY]

# ragged batches with a tight bound of the lengths and without one
_BOUNDED = [(c, True) for c in DECAY] + [(c, False) for c in DECAY if c[1]]
_BOUNDED_IDS = _IDS + [i + "-loose" for i, c in zip(_IDS, DECAY) if c[1]]


def _decay_case(lengths, ragged, H, K, d, dtype, states, g, seed=0, pad=0):
    gen = _gen(seed)
    T, B, n = sum(lengths) + pad, len(lengths), lengths[0]
    act = (lambda h: (h, T, d)) if ragged else (lambda h: (B, h, n, d))
    t = {x: _randn(gen, *act(h), dtype=dtype) for x, h in (("q", H), ("k", K), ("v", K), ("dout", H))}
    t["g"] = torch.tensor(g)
    t["S0"] = _randn(gen, B, K, d, d, scale=2.0) if states else None
    t["dS"] = _randn(gen, B, K, d, d, scale=0.5) if states else None
    t["cu"] = torch.tensor([0] + lengths).cumsum(0).to(torch.int32) if ragged else None
    return t


def _pieces(x, lengths, ragged):
    at = 0
    for s, n in enumerate(lengths):
        yield x[:, at:at + n] if ragged else x[s]
        at += n


def _c(n, d, dtype):
    return (2 * d + 144 + n / 64) * 2 * U + (2.0 ** -16 if dtype == BF16 else 0.0)


@pytest.mark.parametrize("case,tight", _BOUNDED, ids=_BOUNDED_IDS)
def test_decay_forward(case, tight):
    lengths, ragged, H, K, d, dtype, states, g = case
    t = _decay_case(*case)
    scale = d ** -0.5
    out, S = gbla.decay_attention(*_dev(t["q"], t["k"], t["v"], t["g"]), initial_state=_dev(t["S0"])[0],
                                  final_state=True, cu_seqlens=_dev(t["cu"])[0],
                                  max_seqlen=max(lengths) if tight else None)
    assert out.dtype == dtype and S.dtype == F32
    parts = [_pieces(t[x], lengths, ragged) for x in ("q", "k", "v")]
    for s, (q, k, v, y) in enumerate(zip(*parts, _pieces(out, lengths, ragged))):
        S0 = None if t["S0"] is None else t["S0"][s]
        want, final = ref.decay(q, k, v, t["g"], scale, S0)
        size, size_S = ref.decay_sizes(q, k, v, t["g"], scale, S0)
        _check(y, want, size, _c(lengths[s], d, dtype), "out")
        # the state's products have fp32's accuracy for both types
        _check(S[s], final, size_S, (2 * d + 144 + lengths[s] / 64) * 2 * U, "final_state")
        if lengths[s] == 0:
            assert torch.equal(S[s].cpu(), torch.zeros(K, d, d) if S0 is None else S0)


@pytest.mark.parametrize("case,tight", _BOUNDED, ids=_BOUNDED_IDS)
def test_decay_backward(case, tight):
    lengths, ragged, H, K, d, dtype, states, g = case
    t = _decay_case(*case)
    scale = d ** -0.5
    got = gbla.decay_attention_backward(*_dev(t["q"], t["k"], t["v"], t["g"], t["dout"]),
                                        initial_state=_dev(t["S0"])[0], dfinal_state=_dev(t["dS"])[0],
                                        cu_seqlens=_dev(t["cu"])[0],
                                        max_seqlen=max(lengths) if tight else None)
    assert ("dinitial_state" in got) == states
    dg, dg_size = torch.zeros(K).double(), torch.zeros(K).double()
    parts = [_pieces(x, lengths, ragged) for x in
             (t["q"], t["k"], t["v"], t["dout"], got["dq"], got["dk"], got["dv"])]
    for s, (q, k, v, do, dq, dk, dv) in enumerate(zip(*parts)):
        S0, dS = (t["S0"][s], t["dS"][s]) if states else (None, None)
        want = ref.decay_backward(q, k, v, t["g"], do, scale, S0, dS)
        size = ref.decay_backward_sizes(q, k, v, t["g"], do, scale, S0, dS)
        c = _c(lengths[s], d, dtype)
        for name, y, w, z in zip(("dq", "dk", "dv"), (dq, dk, dv), want, size):
            assert y.dtype == dtype
            _check(y, w, z, c, name)
        dg += want[3]
        dg_size += size[3] * c
        if states:
            _check(got["dinitial_state"][s], want[4], size[4], (2 * d + 144 + lengths[s] / 64) * 2 * U,
                   "dinitial_state")
    _check(got["dlog_decay"], dg, dg_size, 1.0, "dlog_decay")


# more sequences than a workgroup has threads, a long one (split into units) among them
_MANY = [([0, 1, 3, 0, 20, 2] * 110)[:count] + [1500, 0, 7] for count in (254, 255, 600)]


@pytest.mark.parametrize("lengths", _MANY, ids=lambda x: str(len(x)))
@pytest.mark.parametrize("dtype,d", [(BF16, 32), (F32, 64)])
def test_decay_many_sequences(lengths, dtype, d):
    case = (lengths, True, 1, 1, d, dtype, True, [-0.01])
    test_decay_forward(case, True)
    test_decay_backward(case, True)


def test_decay_backward_without_the_decay_gradient_and_into_given_outputs():
    t = _decay_case([700], False, 4, 2, 64, BF16, True, [-0.01, -0.1])
    args = _dev(t["q"], t["k"], t["v"], t["g"], t["dout"])
    S0, dS = _dev(t["S0"], t["dS"])
    a = gbla.decay_attention_backward(*args, initial_state=S0, dfinal_state=dS)
    mine = {n: torch.full_like(a[n], 7.0) for n in ("dq", "dk", "dv")}
    mine["dinitial_state"] = dS  # in place
    b = gbla.decay_attention_backward(*args, initial_state=S0, dfinal_state=dS, grads=mine, decay_grad=False)
    assert "dlog_decay" not in b and b["dq"] is mine["dq"] and b["dinitial_state"] is dS
    for n in ("dq", "dk", "dv", "dinitial_state"):
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("n", [100, 900])
def test_decay_state_in_place(n):
    t = _decay_case([n] * 2, False, 4, 2, 64, BF16, True, [-0.01, -0.1])
    args = _dev(t["q"], t["k"], t["v"], t["g"])
    S0, = _dev(t["S0"])
    a, Sa = gbla.decay_attention(*args, initial_state=S0, final_state=True)
    b, Sb = gbla.decay_attention(*args, initial_state=S0, final_state=S0)
    assert Sb is S0 and torch.equal(a, b) and torch.equal(Sa, S0)
    c, none = gbla.decay_attention(*args, initial_state=_dev(t["S0"])[0])
    assert none is None and torch.equal(a, c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths", [[40, 0, 3], [700, 1, 64]])
def test_decay_rows_past_the_last_sequence_are_left(lengths, dtype):
    """Rows behind cu[N]: not read (they are NaN) and not written."""
    t = _decay_case(lengths, True, 4, 2, 64, dtype, False, [-0.01, -0.1], pad=70)
    T = sum(lengths)
    for x in ("q", "k", "v", "dout"):
        t[x][:, T:] = float("nan")
    q, k, v, g, do, cu = _dev(t["q"], t["k"], t["v"], t["g"], t["dout"], t["cu"])
    out = torch.full_like(q, 5.0)
    _, S = gbla.decay_attention(q, k, v, g, cu_seqlens=cu, out=out, final_state=True)
    grads = dict(dq=torch.full_like(q, 5.0), dk=torch.full_like(k, 5.0), dv=torch.full_like(v, 5.0))
    grads = gbla.decay_attention_backward(q, k, v, g, do, cu_seqlens=cu, grads=grads)
    w = torch.ones(4, 64, device="cuda"), torch.ones(2, 64, device="cuda")
    rq, rk = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    gbla.qk_norm_rope(q, k, *w, cu_seqlens=cu, q_out=rq, k_out=rk)
    rg = gbla.qk_norm_rope_backward(q, k, *w, do, v, cu_seqlens=cu,
                                    grads=dict(dq=torch.full_like(q, 5.0), dk=torch.full_like(k, 5.0)))
    for y in (out, grads["dq"], grads["dk"], grads["dv"], rq, rk, rg["dq"], rg["dk"]):
        assert (y[:, T:] == 5.0).all() and torch.isfinite(y).all()
    for y in (S, grads["dlog_decay"], rg["dq_w"], rg["dk_w"]):
        assert torch.isfinite(y).all()


def test_decay_sequences_do_not_reach_each_other():
    """Infinities and NaN in one sequence leave the others' bits alone."""
    lengths = [90, 50, 700, 20]
    t = _decay_case(lengths, True, 2, 2, 64, BF16, True, [-0.01, -0.1])
    q, k, v, g, do, cu, S0, dS = _dev(*(t[x] for x in ("q", "k", "v", "g", "dout", "cu", "S0", "dS")))

    def both():
        out, S = gbla.decay_attention(q, k, v, g, initial_state=S0, final_state=True, cu_seqlens=cu)
        gr = gbla.decay_attention_backward(q, k, v, g, do, initial_state=S0, dfinal_state=dS, cu_seqlens=cu)
        return [out, gr["dq"], gr["dk"], gr["dv"]], [S, gr["dinitial_state"]]

    rows, states = both()
    for x in (q, k, v, do):
        x[:, 90:115] = float("inf")
        x[:, 115:140] = float("nan")
    S0[1] = float("nan")
    rows2, states2 = both()
    for a, b in zip(rows, rows2):
        assert torch.equal(a[:, :90], b[:, :90]) and torch.equal(a[:, 140:], b[:, 140:])
    for a, b in zip(states, states2):
        assert torch.equal(a[[0, 2, 3]], b[[0, 2, 3]])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,dtype", [(300, BF16), (900, BF16), (300, F32)])
def test_decay_nan_stays_behind_its_block_of_tokens(n, dtype, bad):
    t = _decay_case([n], False, 2, 1, 64, dtype, False, [-0.01])
    q, k, v, g, do = _dev(t["q"], t["k"], t["v"], t["g"], t["dout"])
    out, _ = gbla.decay_attention(q, k, v, g)
    gr = gbla.decay_attention_backward(q, k, v, g, do)
    v2, do2 = v.clone(), do.clone()
    v2[:, :, 100] = bad
    do2[:, :, 100] = bad
    out2, _ = gbla.decay_attention(q, k, v2, g)
    assert torch.equal(out[:, :, :64], out2[:, :, :64])
    assert not torch.isfinite(out2[:, :, 100:]).any()
    gr2 = gbla.decay_attention_backward(q, k, v, g, do2)
    for x in ("dk", "dv"):
        assert torch.equal(gr[x][:, :, 128:], gr2[x][:, :, 128:]), x
        assert not torch.isfinite(gr2[x][:, :, :101]).any(), x
    others = [i for i in range(n) if i != 100]
    assert torch.equal(gr["dq"][:, :, others], gr2["dq"][:, :, others])


def test_decay_without_tokens():
    g = torch.tensor([-0.1, -0.2], device="cuda")
    x = torch.empty(3, 2, 0, 64, dtype=BF16, device="cuda")
    S0 = torch.randn(3, 2, 64, 64, device="cuda")
    out, S = gbla.decay_attention(x, x, x, g, initial_state=S0, final_state=True)
    assert out.shape == x.shape and torch.equal(S, S0)
    r = gbla.decay_attention_backward(x, x, x, g, x, initial_state=S0, dfinal_state=S0)
    assert torch.equal(r["dinitial_state"], S0) and (r["dlog_decay"] == 0).all()
    w = torch.ones(2, 64, device="cuda")
    a, b = gbla.qk_norm_rope(x, x, w, w)
    assert a.numel() == b.numel() == 0
    r = gbla.qk_norm_rope_backward(x, x, w, w, x, x)
    assert (r["dq_w"] == 0).all() and (r["dk_w"] == 0).all()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 128), (BF16, 32)])
def test_decay_same_bits_every_time(dtype, d):
    t = _decay_case([900] * 2, False, 4, 2, d, dtype, True, [-0.01, -0.1])
    args = _dev(t["q"], t["k"], t["v"], t["g"])
    do, S0, dS = _dev(t["dout"], t["S0"], t["dS"])
    first = None
    for _ in range(3):
        out, S = gbla.decay_attention(*args, initial_state=S0, final_state=True)
        r = gbla.decay_attention_backward(*args, do, initial_state=S0, dfinal_state=dS)
        now = [out, S] + [r[n] for n in sorted(r)]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_decay_beyond_32_bit_offsets():
    """More than 2^31 elements of q: the last sequence's results are those of its own batch."""
    B, H, n, d = 40, 16, 32768, 128
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free memory")
    g = torch.linspace(-0.05, -0.001, H, device="cuda")
    q = torch.empty(B, H, n, d, dtype=BF16, device="cuda").normal_()
    out, S = gbla.decay_attention(q, q, q, g, final_state=True)
    last = q[B - 1:].clone()
    one, S1 = gbla.decay_attention(last, last, last, g, final_state=True)
    # the batch's and the single sequence's splits differ: a step of bf16 beside the sums' size
    a, b = out[B - 1].float(), one[0].float()
    assert ((a - b).norm() / b.norm()).item() < 2.0 ** -8
    assert ((S[B - 1] - S1[0]).norm() / S1.norm()).item() < 1e-5


# ---------------------------------------------------------------------------
# Single tokens
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,K,d,slots", [(1, 1, 1, 32, None), (3, 8, 2, 64, None), (5, 5, 1, 128, 9),
                                           (300, 2, 2, 32, 301), (2, 12, 1, 64, 2)])
def test_step(N, H, K, d, slots, dtype):
    gen = _gen(1)
    q, k, v = (_randn(gen, N, h, d, dtype=dtype) for h in (H, K, K))
    g = -torch.rand(K, generator=gen)
    state = _randn(gen, slots or N + 1, K, d, d)
    idx = torch.randperm(slots, generator=gen)[:N].to(torch.int32) if slots else None
    S, = _dev(state.clone())
    out = gbla.decay_step(*_dev(q, k, v, g), S, state_indices=_dev(idx)[0])
    rows = idx.tolist() if slots else range(N)
    for n, s in enumerate(rows):
        args = (q[n][:, None], k[n][:, None], v[n][:, None], g, d ** -0.5, state[s])
        want, final = ref.decay(*args)
        size, size_S = ref.decay_sizes(*args)
        _check(out[n], want[:, 0], size[:, 0], (d + 8) * 2 * U, "out")
        _check(S[s], final, size_S, 8 * U, "state")
    left = [s for s in range(state.shape[0]) if s not in set(rows)]
    assert torch.equal(S[left].cpu(), state[left])


def test_step_rows_of_one_slot_follow_each_other_and_others_are_skipped():
    gen = _gen(2)
    N, H, K, d = 7, 4, 2, 64
    q, k, v = (_randn(gen, N, h, d, dtype=BF16) for h in (H, K, K))
    g, state = -torch.rand(K, generator=gen), _randn(gen, 4, K, d, d)
    idx = torch.tensor([2, -1, 2, 0, 4, 2, 2 ** 30], dtype=torch.int32)
    S, = _dev(state.clone())
    out = torch.full((N, H, d), 5.0, dtype=BF16, device="cuda")
    gbla.decay_step(*_dev(q, k, v, g), S, state_indices=_dev(idx)[0], out=out)
    assert (out[[1, 4, 6]] == 5.0).all()
    # the same rows one call each
    S1, = _dev(state.clone())
    for n in (0, 2, 3, 5):
        one = gbla.decay_step(*_dev(q[n:n + 1], k[n:n + 1], v[n:n + 1], g), S1,
                              state_indices=_dev(idx[n:n + 1])[0])
        assert torch.equal(one[0], out[n])
    assert torch.equal(S, S1)
    assert torch.equal(S[[1, 3]].cpu(), state[[1, 3]])


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,n", [(BF16, 90), (F32, 600)])
def test_prompt_then_tokens_is_the_whole_sequence(dtype, n):
    """Norm and rotation, the prompt in chunks with its final state, then single tokens at
    their positions, against the whole sequence in 64 bits."""
    gen = _gen(7)
    B, H, K, d, more = 2, 4, 2, 64, 5
    N = n + more
    q, k, v = (_randn(gen, B, h, N, d, dtype=dtype) for h in (H, K, K))
    q_w, k_w, g = 1 + 0.1 * _randn(gen, H, d), 1 + 0.1 * _randn(gen, K, d), torch.tensor([-0.01, -0.1])
    w = _dev(q_w, k_w)
    cut = lambda x, a, b: x[:, :, a:b].contiguous().cuda()
    qr, kr = gbla.qk_norm_rope(cut(q, 0, n), cut(k, 0, n), *w)
    out, S = gbla.decay_attention(qr, kr, cut(v, 0, n), g.cuda(), final_state=True)
    outs, q_all, k_all = [out], [qr], [kr]
    for t in range(n, N):
        pos = torch.full((B, 1), t, dtype=torch.int32, device="cuda")
        qt, kt = gbla.qk_norm_rope(cut(q, t, t + 1), cut(k, t, t + 1), *w, positions=pos)
        outs.append(gbla.decay_step(qt[:, :, 0], kt[:, :, 0], cut(v, t, t + 1)[:, :, 0], g.cuda(), S)[:, :, None])
        q_all.append(qt), k_all.append(kt)
    got, qx, kx = (torch.cat(x, 2) for x in (outs, q_all, k_all))
    for b in range(B):
        want, final = ref.decay(qx[b].cpu(), kx[b].cpu(), v[b], g, d ** -0.5)
        size, size_S = ref.decay_sizes(qx[b].cpu(), kx[b].cpu(), v[b], g, d ** -0.5)
        _check(got[b], want, size, _c(N, d, dtype), "out")
        _check(S[b], final, size_S, (2 * d + 144 + N / 64 + 8) * 2 * U, "state")
        full = ref.rope(q[b], q_w, torch.arange(N), d)
        _check(qx[b], full, _pair_size(ref.rope(q[b], q_w, torch.arange(N), 0), d, False),
               (d / 8 + 24) * 2 * U, "q")


def test_layer_projections_into_the_decoder():
    """The layer's projections are the operators' inputs as they are."""
    gen = _gen(8)
    B, L, m, H, d = 2, 130, 128, 2, 64
    x = _randn(gen, B, L, m, dtype=BF16).cuda()
    conv = torch.zeros(m, 4, device="cuda")
    conv[:, 3] = 1.0
    p = gbla.layer_project(x, conv, _randn(gen, H * (4 * d + 1), m, dtype=BF16, scale=m ** -0.5).cuda(), H, d)
    w = torch.ones(H, d, device="cuda")
    q, k = gbla.qk_norm_rope(p["q"], p["k"], w, w)
    g = torch.tensor([-0.02, -0.1])
    out, _ = gbla.decay_attention(q, k, p["v"], g.cuda())
    for b in range(B):
        args = (q[b].cpu(), k[b].cpu(), p["v"][b].cpu(), g, d ** -0.5)
        _check(out[b], ref.decay(*args)[0], ref.decay_sizes(*args)[0], _c(L, d, BF16), "out")


@pytest.mark.parametrize("n", [70, 700])
def test_captured_and_replayed_on_another_stream(n):
    """All operators in one captured graph, replayed on new inputs, against eager calls."""
    gen = _gen(9)
    B, H, K, d = 2, 4, 2, 64
    mk = lambda h, m=n: _randn(gen, B, h, m, d, dtype=BF16).cuda()
    t = dict(q=mk(H), k=mk(K), v=mk(K), do=mk(H), S0=_randn(gen, B, K, d, d).cuda())
    w = (1 + 0.1 * _randn(gen, H, d)).cuda(), (1 + 0.1 * _randn(gen, K, d)).cuda()
    g = torch.tensor([-0.01, -0.1], device="cuda")

    def run(S):
        q, k = gbla.qk_norm_rope(t["q"], t["k"], *w)
        out, S = gbla.decay_attention(q, k, t["v"], g, initial_state=S, final_state=S)
        r = gbla.decay_attention_backward(q, k, t["v"], g, t["do"], initial_state=t["S0"])
        e = gbla.qk_norm_rope_backward(t["q"], t["k"], *w, r["dq"], r["dk"])
        y = gbla.decay_step(q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), t["v"][:, :, 0].contiguous(), g, S)
        return [q, k, out, y] + [r[x] for x in sorted(r)] + [e[x] for x in sorted(e)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    S = t["S0"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        run(S)  # warm-up
        with torch.cuda.graph(graph, stream=stream):
            kept = run(S)
    for seed in range(3):
        gen.manual_seed(100 + seed)
        for x in ("q", "k", "v", "do"):
            t[x].copy_(_randn(gen, *t[x].shape, dtype=BF16))
        S.copy_(t["S0"])
        graph.replay()
        torch.cuda.synchronize()
        S1 = t["S0"].clone()
        want = run(S1)
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        assert torch.equal(S, S1)


def test_a_given_stream_is_the_one_that_runs():
    """stream=: scratch and outputs belong to it, so calls in flight on two streams do
    not share memory."""
    t = _decay_case([3000] * 2, False, 4, 2, 64, BF16, False, [-0.01, -0.1])
    args = _dev(t["q"], t["k"], t["v"], t["g"])
    do, = _dev(t["dout"])
    want = gbla.decay_attention_backward(*args, do)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        s = streams[i % 2]
        got.append(gbla.decay_attention_backward(*args, do, stream=s if i < 4 else s.cuda_stream))
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(r[n], want[n]) for n in want)


def test_refuses_what_it_does_not_take():
    t = _decay_case([70] * 2, False, 4, 2, 64, BF16, False, [-0.01, -0.1])
    q, k, v, g = _dev(t["q"], t["k"], t["v"], t["g"])
    with pytest.raises(ValueError, match="contiguous"):
        gbla.decay_attention(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2), g)
    with pytest.raises(TypeError):
        gbla.decay_attention(q, k.float(), v, g)
    with pytest.raises(TypeError):
        gbla.decay_attention(q.half(), k.half(), v.half(), g)
    with pytest.raises(ValueError, match="k has shape"):
        gbla.decay_attention(q, k[:, :, :60].contiguous(), v, g)
    with pytest.raises(ValueError, match="v has shape"):
        gbla.decay_attention(q, k, v[:, :1].contiguous(), g)
    with pytest.raises(ValueError, match="log_decay"):
        gbla.decay_attention(q, k, v, g[:1].clone())
    with pytest.raises(ValueError, match="initial_state"):
        gbla.decay_attention(q, k, v, g, initial_state=torch.zeros(1, 2, 64, 64, device="cuda"))
    with pytest.raises(gbla.GblaError):
        gbla.decay_attention(q[:, :3].contiguous(), k, v, g)      # 2 does not divide 3
    with pytest.raises(ValueError, match="bytes"):
        gbla.decay_attention(q, k, v, g, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="cu_seqlens"):
        gbla.decay_attention(q[0], k[0], v[0], g, cu_seqlens=torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="dout"):
        gbla.decay_attention_backward(q, k, v, g, k)
    w = torch.ones(4, 64, device="cuda"), torch.ones(2, 64, device="cuda")
    with pytest.raises(ValueError, match="k_w"):
        gbla.qk_norm_rope(q, k, w[0], w[0])
    with pytest.raises(ValueError, match="positions"):
        gbla.qk_norm_rope(q, k, *w, positions=torch.zeros(70, dtype=torch.int32, device="cuda"))
    with pytest.raises(gbla.GblaError):
        gbla.qk_norm_rope(q, k, *w, rotary_dim=20)
    S = torch.zeros(2, 2, 64, 64, device="cuda")
    x = q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous()
    with pytest.raises(ValueError, match="state"):
        gbla.decay_step(*x, g, S[:, :1].contiguous())
    with pytest.raises(gbla.GblaError):
        gbla.decay_step(*x, g, S[:1].clone())                     # two rows, one slot
    with pytest.raises(TypeError):
        gbla.decay_step(*x, g, S, state_indices=torch.zeros(2, dtype=torch.int64, device="cuda"))
