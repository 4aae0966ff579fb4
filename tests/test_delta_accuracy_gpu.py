"""How accurate the gated delta rule is, head by head, against the 64-bit recurrence.

Beside the bounds of single entries, which add up absolute values, each head's results are held
to what their type promises, so that no head is judged by the size of another's:

* fp32 results (states, gradients of gates and states, everything in fp32) to 2^-17 of their
  norm.  A result passes a few hundred additions (2 d of products, 128 of a tile's triangle and
  update, the reverse's again) whose roundings, half a step of 2^-24 each, have either sign:
  sqrt(1000) 2^-24 is 2^-19, and a factor of four more for the terms that are larger than their
  sum.
* bf16 results, each off by up to half a step of its type besides, to 2^-8 (1 + 2^-4).
"""
import pytest
import torch

from oracle import gbla_block as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, _dev, _gen, _pieces, _randn
from tests.test_delta_backward_gpu import grads_of
from tests.test_delta_gpu import BOUNDED, BOUNDED_IDS, NAMES, _MANY, delta_case, own, pieces_of, unit
from tests.test_delta_large_gpu import LONG, LONG_IDS

pytestmark = pytest.mark.gpu

TYPES = [(BF16, 32), (BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)]
GRADS = ("dq", "dk", "dv", "dlog_decay", "dbeta")


def per_head(got, want, name, tol=2.0 ** -17):
    """Heads first: the error's norm within tol of the head's own; in bf16, where a wrong entry
    among many is less than the roundings of all, every entry within half a step and 2^-8 of the
    head's root mean square (parts of 2^-16 of terms up to 2^5 times their sum, six deviations)."""
    half = got.dtype == BF16
    if half:
        tol = 2.0 ** -8 * (1 + 2.0 ** -4)
    got, want = got.cpu().double().flatten(1), want.flatten(1)
    off, size = (got - want).norm(dim=1), want.norm(dim=1)
    assert torch.isfinite(got).all() and (off <= tol * size + 1e-30).all(), "%s: off by %s of the heads' norms" % (
        name, ["%.3g" % x for x in off / size])
    if half:
        over = (got - want).abs() - 2.0 ** -8 * (want.abs() * 1.01 + want.square().mean(dim=1, keepdim=True).sqrt())
        assert (over <= 0).all(), "%s: an entry off by %.3g more" % (name, over.max())


def fast(lengths, d, dtype, rates, seed=5):
    """A packed batch with states whose value heads decay by exp(-rate) a token, or nearly so."""
    t = delta_case(lengths, True, len(rates) // 2, len(rates), d, dtype, True, (0,) * len(rates), seed=seed)
    vary = 0.75 + 0.5 * torch.rand(t["g"].shape, generator=_gen(seed + 1))
    t["g"] = -torch.tensor(rates, dtype=F32)[:, None] * vary
    return t


def gradients(t, **how):
    return grads_of(t, initial_state=_dev(t["S0"])[0], dfinal_state=_dev(t["dS"])[0], cu_seqlens=_dev(t["cu"])[0],
                    **how)


@pytest.mark.parametrize("lengths", [[180, 100], [1000, 333]], ids=lambda x: str(x[0]))
@pytest.mark.parametrize("dtype,d", TYPES)
def test_decays_gradient_of_heads_that_forget_fast(dtype, d, lengths):
    """Where exp(g) is small so is dg, while do o and dv v, which go on from token to token, are
    not: their difference would leave an error that does not shrink with the decay."""
    t = fast(lengths, d, dtype, (2.0 ** -6, 0.5, 1.0, 2.0, 4.0, 8.0, 16.0, 30.0))
    got = gradients(t, max_seqlen=max(lengths))
    for s, (args, have) in enumerate(zip(pieces_of(t, NAMES + ("dout",), lengths, True),
                                         pieces_of(got, GRADS, lengths, True))):
        want = ref.delta_backward(*args, d ** -0.5, t["S0"][s], t["dS"][s])
        for x, y, w in zip(GRADS[2:], have[2:], want[2:]):
            per_head(y, w, "%s of %d" % (x, lengths[s]))


@pytest.mark.parametrize("n", [150, 900])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_decays_gradient_of_single_tokens_that_forget(dtype, d, n):
    """Among tokens that keep the state: those that forget nearly all of it have gradients of that
    size to 2^-14 (in bf16 what passes over such a tile comes of states in two parts, 2^-17 each
    and both signs, whose terms are larger than their sum), and those that forget everything 0."""
    t = fast([n], d, dtype, (2.0 ** -6, 2.0 ** -4, 2.0 ** -8, 2.0 ** -6))
    pick = torch.rand(t["g"].shape, generator=_gen(9))
    kinds = {x: (pick > 0.02 * i) & (pick < 0.02 * (i + 1)) for i, x in enumerate((-3.0, -7.0, -12.0, -25.0))}
    for x, at in kinds.items():
        t["g"][at] = x
    t["g"][pick > 0.99] = -float("inf")
    t["g"][(pick > 0.985) & (pick < 0.99)] = -200.0
    got = gradients(t, max_seqlen=n)["dlog_decay"].cpu()
    args = [t[x] for x in NAMES + ("dout",)]
    want = ref.delta_backward(*args, d ** -0.5, t["S0"][0], t["dS"][0])[3]
    per_head(got, want, "dlog_decay")
    assert (got[pick > 0.985] == 0.0).all()
    for x, at in kinds.items():
        off = (got[at].double() - want[at]).norm() / want[at].norm()
        assert off <= 2.0 ** -14, "tokens of decay exp(%g): off by %.3g of their norm" % (x, off)


def by_heads(pieces):
    """The sequences' [heads, ..] next to each other."""
    return torch.cat([x.flatten(1) for x in pieces], dim=1)


def check_case(case, tight, directions):
    """Every result of a case, head by head over its sequences."""
    lengths, ragged, H, V, d, dtype, states, _ = case
    t = delta_case(*case)
    how = dict(initial_state=_dev(t["S0"])[0], cu_seqlens=_dev(t["cu"])[0], max_seqlen=max(lengths) if tight else None)
    start = lambda s: t["S0"][s] if states else None
    if "forward" in directions:
        out, S = own(t, final_state=True, **how)
        want = [ref.delta(*args, d ** -0.5, start(s)) for s, args in enumerate(pieces_of(t, NAMES, lengths, ragged))]
        per_head(by_heads(_pieces(out, lengths, ragged)), by_heads(w[0] for w in want), "out")
        per_head(by_heads(S), by_heads(w[1] for w in want), "final_state")
    if "backward" in directions:
        got = grads_of(t, dfinal_state=_dev(t["dS"])[0], **how)
        want = [ref.delta_backward(*args, d ** -0.5, start(s), t["dS"][s] if states else None)
                for s, args in enumerate(pieces_of(t, NAMES + ("dout",), lengths, ragged))]
        have = list(pieces_of(got, GRADS, lengths, ragged))
        for i, x in enumerate(GRADS):
            per_head(by_heads(h[i] for h in have), by_heads(w[i] for w in want), x)
        if states:
            per_head(by_heads(got["dinitial_state"]), by_heads(w[5] for w in want), "dinitial_state")


MANY = [(lengths, True, 1, 1, d, dtype, True, (-7,)) for lengths in _MANY for dtype, d in ((BF16, 32), (F32, 64))]


@pytest.mark.parametrize("case,tight", BOUNDED, ids=BOUNDED_IDS)
def test_gradients_of_each_head(case, tight):
    check_case(case, tight, ("backward",))


@pytest.mark.parametrize("case", LONG, ids=LONG_IDS)
def test_gradients_of_each_head_in_units_of_several_tiles(case):
    check_case(case, False, ("backward",))


@pytest.mark.parametrize("case", MANY[1:], ids=lambda c: "%d-%d" % (len(c[0]), c[4]))
def test_gradients_of_each_head_of_many_sequences(case):
    check_case(case, True, ("backward",))


def test_gradients_past_two_to_the_31_elements():
    """Of the last sequence of a packed batch whose v ends past element 2^31."""
    H, V, d, last = 2, 4, 128, 300
    T = 2 ** 22 + 333
    gen = torch.Generator("cuda").manual_seed(4)

    def act(heads, one):
        x = torch.empty(heads, T, d, dtype=BF16, device="cuda").normal_(generator=gen)
        if one:
            for h in range(heads):
                x[h] = unit(x[h]).to(BF16)
        return x

    q, k, v, dout = act(H, True), act(H, True), act(V, False), act(V, False)
    g = -torch.exp2(torch.tensor([-6.0, -3.0, 1.0, 3.0], device="cuda"))[:, None] * torch.rand(V, T, generator=gen, device="cuda")
    b = torch.rand(V, T, generator=gen, device="cuda")
    cu = torch.tensor([0, 2 ** 21, T - last, T], device="cuda", dtype=torch.int32)
    got = gbla.delta_attention_backward(q, k, v, g, b, dout, cu_seqlens=cu)
    tail = [x[:, -last:].cpu() for x in (q, k, v, g, b, dout)]
    for x, w in zip(GRADS, ref.delta_backward(*tail, d ** -0.5)):
        per_head(got[x][:, -last:], w, x)
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("case,tight", BOUNDED, ids=BOUNDED_IDS)
def test_outputs_and_states_of_each_head(case, tight):
    """States are fp32 whatever the type: one bf16 part of what forms them, in place of three, would
    leave 2^-9 of their norm."""
    check_case(case, tight, ("forward",))


@pytest.mark.parametrize("case", LONG, ids=LONG_IDS)
def test_outputs_and_states_of_each_head_in_units_of_several_tiles(case):
    check_case(case, False, ("forward",))


@pytest.mark.parametrize("case", MANY, ids=lambda c: "%d-%d" % (len(c[0]), c[4]))
def test_outputs_and_states_of_each_head_of_many_sequences(case):
    check_case(case, True, ("forward",))


def test_outputs_and_states_past_two_to_the_31_elements():
    H, V, d, last = 2, 4, 128, 300
    T = 2 ** 22 + 333
    gen = torch.Generator("cuda").manual_seed(5)
    q, k = (torch.empty(H, T, d, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    for h in range(H):
        q[h], k[h] = unit(q[h]).to(BF16), unit(k[h]).to(BF16)
    v = torch.empty(V, T, d, dtype=BF16, device="cuda").normal_(generator=gen)
    g = -2.0 ** -6 * torch.rand(V, T, generator=gen, device="cuda")
    b = torch.rand(V, T, generator=gen, device="cuda")
    cu = torch.tensor([0, 2 ** 21, T - last, T], device="cuda", dtype=torch.int32)
    out, S = gbla.delta_attention(q, k, v, g, b, final_state=True, cu_seqlens=cu)
    want, final = ref.delta(*(x[:, -last:].cpu() for x in (q, k, v, g, b)), d ** -0.5)
    per_head(out[:, -last:], want, "out")
    per_head(S[2], final, "final_state")
    del out, S
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("rows", [1, 7])
def test_a_step_of_each_head(rows, dtype, d):
    H, V = 2, 4
    t = delta_case([rows], True, H, V, d, dtype, False, (-3, -4, -5, -6), seed=rows)
    step = _dev(*(t[x].transpose(0, 1).contiguous() for x in NAMES))
    state = _randn(_gen(7), rows, V, d, d)
    S, = _dev(state.clone())
    out = gbla.delta_step(*step, S)
    for n in range(rows):
        want, new = ref.delta(*(t[x][:, n:n + 1] for x in NAMES), d ** -0.5, state[n])
        per_head(out[n], want, "out")
        per_head(S[n], new, "state")


def strong(lengths, d, dtype, beta, alike, decay, seed=6):
    """A packed batch with states and strengths from 1 to 2 (or 2 throughout); `alike`: keys a few
    degrees from one another, where a token written with strength 2 is reflected by the next."""
    t = delta_case(lengths, True, 2, 4, d, dtype, True, (0,) * 4, seed=seed)
    gen = _gen(seed + 1)
    t["beta"] = torch.full(t["beta"].shape, 2.0) if beta == 2 else 1.0 + torch.rand(t["beta"].shape, generator=gen)
    t["g"] = -decay * torch.rand(t["g"].shape, generator=gen)
    if alike:
        k = _randn(gen, 2, 1, d) + 0.05 * _randn(gen, *t["k"].shape)
        t["k"] = unit(k).to(dtype)
    return t


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("beta", ["1 to 2", 2])
@pytest.mark.parametrize("decay", [0.0, 2.0 ** -5])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_strengths_above_one(dtype, d, decay, beta, alike):
    """fp32 results to 2^-17 of their norms, as elsewhere; with keys alike and strengths from 1 to 2 to
    2^-14, since a row of the tile's triangle then adds up 64 entries of up to 2, each off by 2^-24, to
    2^-17 of y, y itself is of up to four times the values' size (what the state predicts is), and
    the gradients take two such sums.

    Keys alike and strengths of 2 throughout: 2^-11.  (I + L beta)^-1 then has entries of 2 with signs
    in turn, so that e = (I + L beta)^-1 y is a sum of the tile's tokens that nothing damps, and its
    norm is 2 * 2 * 64 / pi = 81.  L's entries are rounded at least once, 2^-24 of about 1; as a
    matrix of independent entries of that size L's error has a norm of at most 2 sqrt(64) 2^-24 =
    2^-20, and that of e is 81 * 2^-20 * 2 = 2^-12.7 of e.  The triangle that is stored, which
    substitution rounds entry by entry just so, doubles it, 2^-11.7; the reverse's f = du - M^T
    (beta du) takes the transpose of the same with e already off: 2^-10.7 for products of both.
    Their errors are independent: sqrt(2) 2^-11.7, 2^-11.2."""
    lengths = [130, 1, 700]
    t = strong(lengths, d, dtype, beta, alike, decay)
    tol = 2.0 ** (-17 if not alike else -11 if beta == 2 else -14)
    how = dict(initial_state=_dev(t["S0"])[0], cu_seqlens=_dev(t["cu"])[0], max_seqlen=max(lengths))
    out, S = own(t, final_state=True, **how)
    got = grads_of(t, dfinal_state=_dev(t["dS"])[0], **how)
    cut = lambda x, names: list(pieces_of(x, names, lengths, True))
    ins = cut(t, NAMES + ("dout",))
    want = [ref.delta(*a[:5], d ** -0.5, t["S0"][s]) for s, a in enumerate(ins)]
    back = [ref.delta_backward(*a, d ** -0.5, t["S0"][s], t["dS"][s]) for s, a in enumerate(ins)]
    per_head(by_heads(_pieces(out, lengths, True)), by_heads(w[0] for w in want), "out", tol)
    per_head(by_heads(S), by_heads(w[1] for w in want), "final_state", tol)
    have = cut(got, GRADS)
    for i, x in enumerate(GRADS):
        per_head(by_heads(h[i] for h in have), by_heads(w[i] for w in back), x, tol)
    per_head(by_heads(got["dinitial_state"]), by_heads(w[5] for w in back), "dinitial_state", tol)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_steps_of_strength_above_one(dtype, d):
    """Sixty tokens of keys alike and strength 2, one after the other in place."""
    n = 60
    t = strong([n], d, dtype, 2, True, 2.0 ** -5)
    S, = _dev(t["S0"].clone())
    outs = [gbla.delta_step(*_dev(*(t[x][:, i][None].contiguous() for x in NAMES)), S)[0] for i in range(n)]
    want, final = ref.delta(*(t[x] for x in NAMES), d ** -0.5, t["S0"][0])
    per_head(torch.stack(outs, 1), want, "out")
    per_head(S[0], final, "state")


@pytest.mark.parametrize("dtype,d", [(F32, 32), (BF16, 64)])
@pytest.mark.parametrize("with_states", [False, True])
def test_gradients_of_many_long_sequences(dtype, d, with_states):
    """Sequences of more than 64 tiles that a workgroup walks whole (256 heads' sequences in all), with
    heads that forget fast and single tokens that do; three of them against 64 bits."""
    B, V, n = 32, 8, 4200
    gen = torch.Generator("cuda").manual_seed(8)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    q, k = (unit(randn(B, 2, n, d)).to(dtype) for _ in range(2))
    v, dout = randn(B, V, n, d).to(dtype), randn(B, V, n, d).to(dtype)
    rate = torch.exp2(torch.tensor([-8.0, -6.0, -4.0, -3.0, -6.0, 0.0, 2.0, -9.0], device="cuda"))
    g = -rate[:, None] * torch.rand(B, V, n, generator=gen, device="cuda")
    pick = torch.rand(B, V, n, generator=gen, device="cuda")
    g[:, 4][pick[:, 4] < 0.005] = -9.0
    g[:, 7][pick[:, 7] < 0.001] = -float("inf")
    b = torch.rand(B, V, n, generator=gen, device="cuda")
    S0, dS = (randn(B, V, d, d), randn(B, V, d, d)) if with_states else (None, None)
    got = gbla.delta_attention_backward(q, k, v, g, b, dout, initial_state=S0, dfinal_state=dS)
    at = (0, 17, B - 1)
    want = [ref.delta_backward(*(x[s].cpu() for x in (q, k, v, g, b, dout)), d ** -0.5,
                               *((S0[s].cpu(), dS[s].cpu()) if with_states else (None, None))) for s in at]
    for i, x in enumerate(GRADS):
        per_head(by_heads(got[x][s].cpu() for s in at), by_heads(w[i] for w in want), x)
    dg = got["dlog_decay"]
    assert (dg[torch.isneginf(g)] == 0.0).all()
