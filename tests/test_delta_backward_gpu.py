"""The gated delta rule's backward on the GPU against the 64-bit recurrence's.

Every entry within c sizes (oracle.gbla_block.delta_backward_sizes) and half a step of its type,
c as for the forward with the reverse's additions too: (4 d + 416 + n / 32) 2 u, and 6 * 2^-16
more where a bf16 gradient is formed from products of two parts (each factor's part, the product
of the smaller parts).  Those bounds add up absolute values along the sequence; beside them the
whole of a gradient is held to what its type promises: fp32 ones to 2^-17 of their norm,
bf16 ones, whose entries are each off by up to half a step of 2^-8, to 2^-8 (1 + 2^-4).
"""
import pytest
import torch

from oracle import gbla_block as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, U, _check, _dev, _gen, _pieces
from tests.test_delta_gpu import BOUNDED, BOUNDED_IDS, NAMES, _MANY, delta_case, pieces_of, unit

pytestmark = pytest.mark.gpu


def c_of(n, d):
    return (4 * d + 416 + n / 32) * 2 * U


def grads_of(t, **how):
    return gbla.delta_attention_backward(*_dev(*(t[x] for x in NAMES + ("dout",))), **how)


def whole(got, want, name):
    got = got.cpu().double()
    tol = 2.0 ** -8 * (1 + 2.0 ** -4) if name[1] in "qkv" and name[-1] == "b" else 2.0 ** -17
    assert (got - want).norm() <= tol * want.norm() + 1e-30, "%s off by %.3g of its norm" % (
        name, (got - want).norm() / want.norm())


@pytest.mark.parametrize("case,tight", BOUNDED, ids=BOUNDED_IDS)
def test_delta_backward(case, tight):
    lengths, ragged, H, V, d, dtype, states, _ = case
    t = delta_case(*case)
    scale = d ** -0.5
    got = grads_of(t, initial_state=_dev(t["S0"])[0], dfinal_state=_dev(t["dS"])[0], cu_seqlens=_dev(t["cu"])[0],
                   max_seqlen=max(lengths) if tight else None)
    assert ("dinitial_state" in got) == states
    names = ("dq", "dk", "dv", "dlog_decay", "dbeta")
    mark = "b" if dtype == BF16 else "f"
    total = {x: ([], []) for x in names}
    outs = pieces_of(got, names, lengths, ragged)
    for s, (args, have) in enumerate(zip(pieces_of(t, NAMES + ("dout",), lengths, ragged), outs)):
        S0, dS = (t["S0"][s], t["dS"][s]) if states else (None, None)
        want = ref.delta_backward(*args, scale, S0, dS)
        size = ref.delta_backward_sizes(*args, scale, S0, dS)
        c = c_of(lengths[s], d)
        for x, y, w, z in zip(names, have, want, size):
            assert y.dtype == (dtype if x in ("dq", "dk", "dv") else F32)
            _check(y, w, z, c + (6 * 2.0 ** -16 if y.dtype == BF16 else 0.0), x)
            total[x][0].append(y.cpu().reshape(-1)), total[x][1].append(w.reshape(-1))
        if states:
            _check(got["dinitial_state"][s], want[5], size[5], c, "dinitial_state")
    for x in names:
        whole(torch.cat(total[x][0]), torch.cat(total[x][1]), x + (mark if x in ("dq", "dk", "dv") else "f"))


@pytest.mark.parametrize("lengths", _MANY[1:], ids=lambda x: str(len(x)))
def test_delta_backward_many_sequences(lengths):
    test_delta_backward((lengths, True, 1, 1, 32, BF16, True, (-7,)), True)


@pytest.mark.parametrize("given", ["S0", "dS", "none"])
@pytest.mark.parametrize("n", [90, 700])
def test_delta_backward_with_one_state_or_none(given, n):
    d = 64
    t = delta_case([n], False, 1, 2, d, F32, True, (-4, -7))
    S0, dS = (t["S0"] if given == "S0" else None), (t["dS"] if given == "dS" else None)
    got = grads_of(t, initial_state=_dev(S0)[0], dfinal_state=_dev(dS)[0])
    args = [t[x][0] for x in NAMES + ("dout",)]
    a, b = (None if x is None else x[0] for x in (S0, dS))
    want = ref.delta_backward(*args, d ** -0.5, a, b)
    size = ref.delta_backward_sizes(*args, d ** -0.5, a, b)
    for x, w, z in zip(("dq", "dk", "dv", "dlog_decay", "dbeta", "dinitial_state"), want, size):
        if x in got:
            _check(got[x][0], w, z, c_of(n, d), x)
            whole(got[x][0], w, x + "f")


def test_delta_gradients_are_differences():
    """Central differences of the forward itself, in directions: fp32, so steps of 2^-7 leave
    about 2^-14 (their square) and 2^-24 / 2^-7 of the loss's terms."""
    n, V, d = 150, 2, 32
    t = delta_case([n], False, 1, V, d, F32, True, (-4, -6), seed=3)
    t["g"].clamp_(min=-5.0)
    names = NAMES + ("S0",)
    x = {m: t[m].cuda() for m in names}
    do, dS = t["dout"].cuda(), t["dS"].cuda()

    def loss(y):
        out, S = gbla.delta_attention(*(y[m] for m in NAMES), initial_state=y["S0"], final_state=True)
        return (out.double() * do).sum() + (S.double() * dS).sum()

    got = gbla.delta_attention_backward(*(x[m] for m in NAMES), do, initial_state=x["S0"], dfinal_state=dS)
    have = dict(zip(names, (got[m] for m in ("dq", "dk", "dv", "dlog_decay", "dbeta", "dinitial_state"))))
    for i, m in enumerate(names):
        way = torch.randn(x[m].shape, generator=_gen(20 + i)).cuda()
        way = way * x[m].norm() / way.norm()
        step = 2.0 ** -7
        up, down = dict(x), dict(x)
        up[m], down[m] = x[m] + step * way, x[m] - step * way
        if m == "g":  # stays a decay
            up[m], down[m] = x[m] + step * x[m] * way.sign(), x[m] - step * x[m] * way.sign()
            way = x[m] * way.sign()
        slope = (loss(up) - loss(down)) / (2 * step)
        want = (have[m].double() * way).sum()
        terms = (have[m].double() * way).norm() + loss(x).abs()
        assert (slope - want).abs() <= 2.0 ** -9 * terms, m


def test_delta_backward_into_given_outputs_and_repeated():
    t = delta_case([700], False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    S0, dS = _dev(t["S0"], t["dS"])
    a = grads_of(t, initial_state=S0, dfinal_state=dS)
    mine = {n: torch.full_like(x, 7.0) for n, x in a.items()}
    mine["dinitial_state"] = dS  # in place
    b = grads_of(t, initial_state=S0, dfinal_state=dS, grads=mine)
    assert b["dq"] is mine["dq"] and b["dinitial_state"] is dS
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("lengths", [[40, 0, 3], [700, 1, 64]])
def test_delta_backward_rows_past_the_last_sequence_are_left(lengths):
    t = delta_case(lengths, True, 2, 4, 64, BF16, False, (-5, -6, -7, -8), pad=70)
    T = sum(lengths)
    for x in NAMES + ("dout",):
        t[x][:, T:] = float("nan")
    like = dict(dq="q", dk="k", dv="v", dlog_decay="g", dbeta="beta")
    mine = {n: torch.full_like(t[x], 7.0).cuda() for n, x in like.items()}
    grads_of(t, cu_seqlens=_dev(t["cu"])[0], grads=mine)
    for n, x in mine.items():
        assert (x[:, T:] == 7.0).all() and torch.isfinite(x[:, :T].float()).all(), n


def test_delta_backward_values_that_are_not_finite_stay_in_their_sequence_and_head():
    t = delta_case([200] * 2, False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    how = dict(initial_state=_dev(t["S0"])[0], dfinal_state=_dev(t["dS"])[0])
    want = grads_of(t, **how)
    for x, h in (("q", 1), ("v", 2), ("dout", 3)):
        bad = dict(t)
        bad[x] = t[x].clone()
        bad[x][1, h, 130, 5] = float("nan")
        got = grads_of(bad, **how)
        for n in want:
            heads = [0] if want[n].shape[1] == 2 else [0, 1]
            assert torch.equal(got[n][0], want[n][0]) and torch.equal(got[n][1, heads], want[n][1, heads]), (x, n)


def test_delta_backward_replayed_from_a_graph():
    t = delta_case([1200], False, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    args = _dev(*(t[x] for x in NAMES + ("dout",)))
    S0, dS = _dev(t["S0"], t["dS"])
    shape = gbla.delta_shape(*args[:3])
    ws = torch.empty(gbla.delta_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    how = dict(initial_state=S0, dfinal_state=dS)
    mine = gbla.delta_attention_backward(*args, workspace=ws, **how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gbla.delta_attention_backward(*args, workspace=ws, grads=mine, **how)
    for i in range(3):
        args[5].copy_(torch.randn(args[5].shape, generator=_gen(i)).to(BF16))
        ws.fill_(255)  # whatever the scratch holds
        for x in mine.values():
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = gbla.delta_attention_backward(*args, **how)
        for n in want:
            assert torch.equal(mine[n], want[n]), n
