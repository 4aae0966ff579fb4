"""The gated delta rule on the GPU against the 64-bit recurrence.

Tolerances are bounds, not fits.  With u = 2^-24 (half a step of fp32) and the sizes of
oracle.gbla_block.delta_sizes, which say what a relative error in every term of a tile can add
up to (keys of length at most one, strengths within [0, 1]):

* a term passes at most d (scores or predictions) + 64 + 64 (the triangle's substitution and
  product) + d (the state's read) + 64 (a tile's update) additions, one more for every tile
  and unit that the state is carried over and 16 other roundings; a matrix unit may truncate
  where an addition rounds, hence c = (2 d + 208 + n / 64) 2 u for states and fp32 outputs.
  Three bf16 parts leave 2^-24 of a term, which the truncations' share covers.
* a bf16 output is formed from two parts of the state, the scores and u: each leaves 2^-16 of
  a term (half a step of half a step), and the product of the smaller parts, 2^-16, is left
  out: 4 * 2^-16 more, and half a step of its type.
* a step adds d + 16 roundings a product, d at a time: the same c.
"""
import pytest
import torch

from oracle import gbla_block as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, U, _check, _dev, _gen, _pieces, _randn

pytestmark = pytest.mark.gpu

DELTA = [
    # lengths, ragged, H, V, d, dtype, states, log2 of the decays' rates
    ([1], False, 1, 1, 32, F32, False, (-3,)),
    ([63] * 2, False, 2, 2, 64, BF16, True, (-3, -7)),
    ([64], False, 1, 2, 128, BF16, False, (-2, -9)),
    ([65], False, 1, 4, 128, F32, True, (-4, 2, -9, -6)),
    ([200] * 3, False, 3, 6, 32, BF16, True, (-3, -4, -5, -6, 3, -8)),
    ([257], False, 2, 2, 32, F32, False, (-5, -8)),
    ([600], False, 2, 2, 64, BF16, True, (-6, -9)),
    ([777] * 2, False, 2, 4, 64, F32, True, (-4, -5, -7, -30)),
    ([513], False, 3, 3, 128, BF16, True, (-5, -6, -7)),
    ([640], False, 2, 2, 128, F32, False, (-5, -8)),
    ([1300], False, 1, 2, 32, BF16, False, (-6, -9)),
    ([5, 0, 130, 1, 64, 300], True, 2, 4, 64, F32, True, (-3, -5, -7, -9)),
    ([700, 0, 1, 128, 513], True, 1, 2, 64, BF16, True, (-5, -8)),
    ([0, 900, 64, 0], True, 2, 2, 128, BF16, False, (-5, -8)),
    ([33] * 40, True, 8, 8, 32, BF16, False, tuple(range(-3, -11, -1))),
    ([64, 66] * 20, True, 1, 2, 32, F32, True, (-4, -7)),
]
IDS = ["%s-%s" % ("ragged" if c[1] else "dense", "-".join(map(str, (len(c[0]), max(c[0])) + c[2:7]))) for c in DELTA]
# ragged batches with a tight bound of the lengths and without one
BOUNDED = [(c, True) for c in DELTA] + [(c, False) for c in DELTA if c[1]]
BOUNDED_IDS = IDS + [i + "-loose" for i, c in zip(IDS, DELTA) if c[1]]


def unit(x):
    """Rows a little shorter than one, so that their roundings are at most one long."""
    return 0.99 * x / x.float().norm(dim=-1, keepdim=True).clamp(min=1e-6)


def delta_case(lengths, ragged, H, V, d, dtype, states, rates, seed=0, pad=0):
    gen = _gen(seed)
    T, B, n = sum(lengths) + pad, len(lengths), lengths[0]
    act = (lambda h: (h, T, d)) if ragged else (lambda h: (B, h, n, d))
    t = dict(q=unit(_randn(gen, *act(H))).to(dtype), k=unit(_randn(gen, *act(H))).to(dtype),
             v=_randn(gen, *act(V), dtype=dtype), dout=_randn(gen, *act(V), dtype=dtype))
    gates = act(V)[:-1]
    rate = torch.exp2(torch.tensor(rates, dtype=F32))[:, None]
    t["g"] = -rate * torch.nn.functional.softplus(2.0 * _randn(gen, *gates))
    t["beta"] = torch.sigmoid(2.0 * _randn(gen, *gates))
    # decays and strengths at their ends: nothing kept, all kept, nothing written, all corrected
    pick = torch.rand(gates, generator=gen)
    t["g"][pick < 0.01] = -float("inf")
    t["g"][(pick > 0.02) & (pick < 0.05)] = 0.0
    t["beta"][(pick > 0.05) & (pick < 0.08)] = 0.0
    t["beta"][(pick > 0.08) & (pick < 0.11)] = 1.0
    t["S0"] = _randn(gen, B, V, d, d) if states else None
    t["dS"] = _randn(gen, B, V, d, d, scale=0.5) if states else None
    t["cu"] = torch.tensor([0] + lengths).cumsum(0).to(torch.int32) if ragged else None
    return t


def pieces_of(t, names, lengths, ragged):
    """The sequences' views: the gates have no channels, and are taken as heads of one."""
    cut = {x: list(_pieces(t[x] if t[x].dim() == (3 if ragged else 4) else t[x][..., None], lengths, ragged))
           for x in names}
    for s in range(len(lengths)):
        yield tuple(cut[x][s] if t[x].dim() == (3 if ragged else 4) else cut[x][s][..., 0] for x in names)


def c_of(n, d):
    return (2 * d + 208 + n / 64) * 2 * U


def own(t, **how):
    return gbla.delta_attention(*_dev(t["q"], t["k"], t["v"], t["g"], t["beta"]), **how)


NAMES = ("q", "k", "v", "g", "beta")


@pytest.mark.parametrize("case,tight", BOUNDED, ids=BOUNDED_IDS)
def test_delta_forward(case, tight):
    lengths, ragged, H, V, d, dtype, states, _ = case
    t = delta_case(*case)
    scale = d ** -0.5
    out, S = own(t, initial_state=_dev(t["S0"])[0], final_state=True, cu_seqlens=_dev(t["cu"])[0],
                 max_seqlen=max(lengths) if tight else None)
    assert out.dtype == dtype and S.dtype == F32
    for s, (args, y) in enumerate(zip(pieces_of(t, NAMES, lengths, ragged), _pieces(out, lengths, ragged))):
        S0 = None if t["S0"] is None else t["S0"][s]
        want, final = ref.delta(*args, scale, S0)
        size, size_S = ref.delta_sizes(*args, scale, S0)
        c = c_of(lengths[s], d)
        _check(y, want, size, c + (2.0 ** -14 if dtype == BF16 else 0.0), "out")
        _check(S[s], final, size_S.expand_as(final), c, "final_state")
        if lengths[s] == 0:
            assert torch.equal(S[s].cpu(), torch.zeros(V, d, d) if S0 is None else S0)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 32), (BF16, 128)])
def test_delta_of_equal_keys_and_full_strength(dtype, d):
    """All keys alike and strength one, without decay: the triangle's inverse by powers would
    cancel; the state holds the last value at that key."""
    n = 130
    gen = _gen(1)
    k = unit(_randn(gen, 1, 1, 1, d)).to(dtype).expand(1, 1, n, d).contiguous()
    t = dict(q=k, k=k, v=_randn(gen, 1, 1, n, d, dtype=dtype), g=torch.zeros(1, 1, n), beta=torch.ones(1, 1, n))
    out, S = own(t, scale=1.0, final_state=True)
    want, final = ref.delta(*(t[x][0] for x in NAMES), 1.0)
    size, size_S = ref.delta_sizes(*(t[x][0] for x in NAMES), 1.0)
    _check(out[0], want, size, c_of(n, d) + (2.0 ** -14 if dtype == BF16 else 0.0), "out")
    _check(S[0], final, size_S.expand_as(final), c_of(n, d), "final_state")


# more sequences than a workgroup has threads, a long one (split into units) among them
_MANY = [([0, 1, 3, 0, 20, 2] * 110)[:count] + [1500, 0, 7] for count in (254, 255, 600)]


@pytest.mark.parametrize("lengths", _MANY, ids=lambda x: str(len(x)))
@pytest.mark.parametrize("dtype,d", [(BF16, 32), (F32, 64)])
def test_delta_many_sequences(lengths, dtype, d):
    test_delta_forward((lengths, True, 1, 1, d, dtype, True, (-7,)), True)


@pytest.mark.parametrize("n", [100, 900])
def test_delta_state_in_place(n):
    t = delta_case([n] * 2, False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    S0, = _dev(t["S0"])
    a, Sa = own(t, initial_state=S0, final_state=True)
    b, Sb = own(t, initial_state=S0, final_state=S0)
    assert Sb is S0 and torch.equal(a, b) and torch.equal(Sa, S0)
    c, none = own(t, initial_state=_dev(t["S0"])[0])
    assert none is None and torch.equal(a, c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths", [[40, 0, 3], [700, 1, 64]])
def test_delta_rows_past_the_last_sequence_are_left(lengths, dtype):
    """Rows behind cu[N]: not read (they are NaN) and not written."""
    t = delta_case(lengths, True, 2, 4, 64, dtype, False, (-5, -6, -7, -8), pad=70)
    T = sum(lengths)
    for x in ("q", "k", "v", "g", "beta"):
        t[x][:, T:] = float("nan")
    out = torch.full_like(t["v"], 7.0).cuda()
    own(t, cu_seqlens=_dev(t["cu"])[0], out=out, final_state=True)
    assert (out[:, T:] == 7.0).all() and torch.isfinite(out[:, :T].float()).all()


@pytest.mark.parametrize("n", [70, 700])
@pytest.mark.parametrize("what", ["k", "v", "g", "beta", "q", "+g"])
def test_delta_values_that_are_not_finite(what, n):
    """They reach their own and later outputs of their sequence and heads, and no others."""
    case = ([n] * 2, False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    t = delta_case(*case)
    t["g"].clamp_(min=-20.0)  # no token that forgets
    S0, = _dev(t["S0"])
    want, Sw = own(t, initial_state=S0, final_state=True)
    at, h = n - 45, 1
    bad = float("nan") if what in ("v", "beta") else float("inf")
    if what in ("q", "k", "v"):
        t[what][1, h, at, 5] = bad
    else:
        t[what.strip("+")][1, h, at] = bad
    out, S = own(t, initial_state=S0, final_state=True)
    heads = [2, 3] if what in ("q", "k") else [1]
    mine = torch.zeros_like(out, dtype=torch.bool)
    mine[1, heads, at:(at + 1 if what == "q" else n)] = True
    assert torch.isnan(out[mine]).all() and torch.equal(out[~mine], want[~mine])
    lost = torch.zeros_like(S, dtype=torch.bool)
    lost[1, heads] = what != "q"
    assert torch.isnan(S[lost]).all() and torch.equal(S[~lost], Sw[~lost])


def test_delta_a_token_without_memory_forgets_the_state():
    """log_decay -inf: the outputs from that token on are those of a sequence that starts there."""
    t = delta_case([300], False, 2, 2, 64, F32, True, (-5, -6))
    t["g"].clamp_(min=-20.0)
    t["g"][:, :, 130] = -float("inf")
    out, S = own(t, initial_state=_dev(t["S0"])[0], final_state=True)
    late = {x: t[x][:, :, 130:].contiguous() for x in NAMES}
    want, Sw = own(late, final_state=True)
    args = [late[x][0] for x in NAMES]
    size, size_S = ref.delta_sizes(*args, 64 ** -0.5)
    assert ((out[:, :, 130:] - want).abs().cpu()[0] <= 2 * c_of(300, 64) * size).all()
    assert ((S - Sw).abs().cpu()[0] <= 2 * c_of(300, 64) * size_S).all()


@pytest.mark.parametrize("H,V,d,dtype", [(1, 1, 32, F32), (2, 4, 64, BF16), (4, 4, 64, F32), (2, 8, 128, BF16),
                                         (3, 3, 128, F32), (2, 2, 32, BF16)])
@pytest.mark.parametrize("rows", [1, 5])
def test_delta_step(rows, H, V, d, dtype):
    """Against the recurrence; the same slot twice, slots out of range, states of others left."""
    rates = tuple(-3 - i for i in range(V))
    t = delta_case([rows], True, H, V, d, dtype, False, rates, seed=rows)
    step = {x: t[x].transpose(0, 1).contiguous() for x in NAMES}  # [rows, heads, ..]
    slots = 4
    state = _randn(_gen(7), slots, V, d, d)
    index = torch.tensor([2, 0, 2, -1, slots][:rows], dtype=torch.int32)
    out = torch.full((rows, V, d), 7.0, dtype=dtype).cuda()
    S, = _dev(state.clone())
    got = gbla.delta_step(*_dev(*(step[x] for x in NAMES)), S, state_indices=index.cuda(), out=out)
    assert got is out
    now = state.clone().double()
    size = torch.zeros(slots, V, 1, d, dtype=torch.float64)
    for n, s in enumerate(index.tolist()):
        if not 0 <= s < slots:
            assert (out[n] == 7.0).all()
            continue
        args = [step[x][n][:, None] for x in NAMES]
        want, new = ref.delta(*args, d ** -0.5, now[s])
        so, sS = ref.delta_sizes(*args, d ** -0.5, now[s])
        size[s] += sS
        _check(out[n], want[:, 0], so[:, 0] + d ** -0.5 * size[s][:, 0], c_of(rows, d), "out %d" % n)
        now[s] = new
    for s in range(slots):
        if s in index.tolist():
            _check(S[s], now[s], size[s].expand_as(now[s]), c_of(rows, d), "state")
        else:
            assert torch.equal(S[s].cpu(), state[s])


def test_delta_step_without_indices():
    t = delta_case([3], True, 1, 2, 64, BF16, False, (-4, -6))
    step = _dev(*(t[x].transpose(0, 1).contiguous() for x in NAMES))
    a, b = (_randn(_gen(7), 5, 2, 64, 64).cuda() for _ in range(2))
    x = gbla.delta_step(*step, a)
    y = gbla.delta_step(*step, b, state_indices=torch.arange(3, dtype=torch.int32, device="cuda"))
    assert torch.equal(x, y) and torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_delta_prompt_then_tokens_is_the_whole_sequence(dtype):
    n, more, V, d = 200, 3, 4, 64
    t = delta_case([n + more] * 2, False, 2, V, d, dtype, False, (-5, -6, -7, -8))
    q, k, v, g, b = _dev(*(t[x] for x in NAMES))
    head = [x[:, :, :n].contiguous() for x in (q, k, v, g, b)]
    out, S = gbla.delta_attention(*head, final_state=True)
    outs = [out]
    for i in range(n, n + more):
        outs.append(gbla.delta_step(*(x[:, :, i].contiguous() for x in (q, k, v, g, b)), S)[:, :, None])
    got = torch.cat(outs, dim=2)
    for s in range(2):
        args = [t[x][s] for x in NAMES]
        want, final = ref.delta(*args, d ** -0.5)
        size, size_S = ref.delta_sizes(*args, d ** -0.5)
        _check(got[s], want, size, c_of(n, d) + (2.0 ** -14 if dtype == BF16 else 0.0), "out")
        _check(S[s], final, size_S.expand_as(final), c_of(n, d), "state")


@pytest.mark.parametrize("lengths", [[150] * 2, [1200]])
def test_delta_replayed_from_a_graph_and_on_another_stream(lengths):
    """One workspace for two captured calls, eager work between the replays."""
    t = delta_case(lengths, False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    q, k, v, g, b, S0 = _dev(*(t[x] for x in NAMES), t["S0"])
    shape = gbla.delta_shape(q, k, v)
    ws = torch.empty(gbla.delta_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    call = lambda x, y: gbla.delta_attention(q, k, x, g, b, initial_state=S0, final_state=y[1], workspace=ws, out=y[0])
    v2 = (v * 0.5).contiguous()
    bufs = [(torch.empty_like(v), torch.empty_like(S0)) for _ in range(2)]
    call(v, bufs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(v, bufs[0])
        call(v2, bufs[1])
    for i in range(3):
        v.copy_(torch.randn(v.shape, generator=_gen(i)).to(v.dtype))
        v2.copy_(v)
        for y in bufs:
            y[0].zero_(), y[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, Sw = gbla.delta_attention(q, k, v, g, b, initial_state=S0, final_state=True)
        for y in bufs:
            assert torch.equal(y[0], want) and torch.equal(y[1], Sw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, S = gbla.delta_attention(q, k, v, g, b, initial_state=S0, final_state=True, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(S, Sw)


def test_delta_repeated_calls_give_the_same_bits():
    t = delta_case([900, 3, 1500], True, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    how = dict(initial_state=_dev(t["S0"])[0], final_state=True, cu_seqlens=_dev(t["cu"])[0], max_seqlen=1500)
    a, Sa = own(t, **how)
    b, Sb = own(t, **how)
    assert torch.equal(a, b) and torch.equal(Sa, Sb)


def test_delta_refuses_tensors():
    t = delta_case([20], False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    q, k, v, g, b, S0 = _dev(*(t[x] for x in NAMES), t["S0"])
    ok = dict(q=q, k=k, v=v, log_decay=g, beta=b)
    wrong = [dict(k=k[:, :1].contiguous()), dict(v=v[:, :3].contiguous()), dict(log_decay=g.bfloat16()),
             dict(beta=b[:, :2].contiguous()), dict(v=v.transpose(1, 2)), dict(q=q.float()), dict(beta=b.cpu()),
             dict(initial_state=S0[:, :2].contiguous()), dict(out=torch.empty_like(q)), dict(final_state=S0[0]),
             dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))]
    for change in wrong:
        with pytest.raises((ValueError, TypeError, gbla.GblaError)):
            gbla.delta_attention(**{**ok, **change})
    assert gbla.delta_attention(**ok)[0].shape == v.shape
