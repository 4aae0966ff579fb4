"""The gated delta rule and the residual norm at sizes: units of several tiles, sequences of a
hundred thousand tokens, arrays of more than 2^31 elements, two streams at once.

Against the 64-bit recurrence the tolerances are those of the small cases (their derivation is
beside them).  A whole against the same tokens in pieces: either is within 2^-17 of the exact
result's norm, so the two are within 2^-16 of each other.
"""
import pytest
import torch

from oracle import gbla_block as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, _check, _dev, _pieces
from tests.test_delta_backward_gpu import c_of as c_back
from tests.test_delta_backward_gpu import grads_of
from tests.test_delta_gpu import NAMES, c_of, delta_case, own, pieces_of, unit

pytestmark = pytest.mark.gpu

# lengths, ragged, H, V, d, dtype, states, log2 of the rates: units of 128 and 256 tokens
LONG = [
    ([4500, 130, 5000], True, 4, 8, 64, BF16, True, tuple(range(-3, -11, -1))),
    ([4200], False, 8, 8, 32, F32, False, tuple(range(-3, -11, -1))),
    ([4200], False, 4, 8, 128, BF16, True, tuple(range(-3, -11, -1))),
]
LONG_IDS = ["%d-%d" % (max(c[0]), c[4]) for c in LONG]


@pytest.mark.parametrize("case", LONG, ids=LONG_IDS)
def test_delta_units_of_several_tiles(case):
    lengths, ragged, H, V, d, dtype, states, _ = case
    t = delta_case(*case)
    scale = d ** -0.5
    out, S = own(t, initial_state=_dev(t["S0"])[0], final_state=True, cu_seqlens=_dev(t["cu"])[0])
    for s, (args, y) in enumerate(zip(pieces_of(t, NAMES, lengths, ragged), _pieces(out, lengths, ragged))):
        S0 = t["S0"][s] if states else None
        want, final = ref.delta(*args, scale, S0)
        size, size_S = ref.delta_sizes(*args, scale, S0)
        c = c_of(lengths[s], d)
        _check(y, want, size, c + (2.0 ** -14 if dtype == BF16 else 0.0), "out")
        _check(S[s], final, size_S.expand_as(final), c, "final_state")


@pytest.mark.parametrize("case", LONG, ids=LONG_IDS)
def test_delta_backward_units_of_several_tiles(case):
    lengths, ragged, H, V, d, dtype, states, _ = case
    t = delta_case(*case)
    scale = d ** -0.5
    got = grads_of(t, initial_state=_dev(t["S0"])[0], dfinal_state=_dev(t["dS"])[0], cu_seqlens=_dev(t["cu"])[0])
    names = ("dq", "dk", "dv", "dlog_decay", "dbeta")
    for s, (args, have) in enumerate(zip(pieces_of(t, NAMES + ("dout",), lengths, ragged),
                                         pieces_of(got, names, lengths, ragged))):
        S0, dS = (t["S0"][s], t["dS"][s]) if states else (None, None)
        want = ref.delta_backward(*args, scale, S0, dS)
        size = ref.delta_backward_sizes(*args, scale, S0, dS)
        c = c_back(lengths[s], d)
        for x, y, w, z in zip(names, have, want, size):
            _check(y, w, z, c + (6 * 2.0 ** -16 if y.dtype == BF16 else 0.0), x)


def near(a, b, name):
    # (bf16 entries are off by half a step each besides)
    tol = 2.0 ** -16 if a.dtype == F32 else 2.0 ** -7
    a, b = a.double(), b.double()
    assert torch.isfinite(a).all() and (a - b).norm() <= tol * b.norm(), "%s off by %.3g of its norm" % (
        name, (a - b).norm() / b.norm())


@pytest.mark.parametrize("dtype,d,n", [(F32, 32, 131072 + 77), (BF16, 64, 40000)])
def test_delta_of_a_long_sequence_is_its_pieces(dtype, d, n):
    """Units of 512 and 1024 tokens against pieces of other sizes, each with the state and the
    gradient of the state that its neighbour leaves."""
    H, V, cuts = 4, 8, (0, n // 3, n // 2 + 5, n)
    gen = torch.Generator("cuda").manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    args = [unit(randn(1, H, n, d)).to(dtype), unit(randn(1, H, n, d)).to(dtype), randn(1, V, n, d).to(dtype),
            -torch.exp2(-torch.arange(3.0, 3 + V, device="cuda"))[:, None] * randn(1, V, n).abs(),
            torch.rand(1, V, n, generator=gen, device="cuda")]
    dout, dS = randn(1, V, n, d).to(dtype), randn(1, V, d, d)
    S0 = randn(1, V, d, d)
    piece = lambda i: [x[:, :, cuts[i]:cuts[i + 1]].contiguous() for x in args + [dout]]
    out, S = gbla.delta_attention(*args, initial_state=S0, final_state=True)
    states = [S0]
    for i in range(3):
        y, state = gbla.delta_attention(*piece(i)[:5], initial_state=states[-1], final_state=True)
        states.append(state)
        near(out[:, :, cuts[i]:cuts[i + 1]], y, "out")
    near(S, states[-1], "final_state")
    got = gbla.delta_attention_backward(*args, dout, initial_state=S0, dfinal_state=dS)
    for i in (2, 1, 0):
        g = gbla.delta_attention_backward(*piece(i), initial_state=states[i], dfinal_state=dS)
        dS = g["dinitial_state"]
        for x in ("dq", "dk", "dv", "dlog_decay", "dbeta"):
            near(got[x][:, :, cuts[i]:cuts[i + 1]], g[x], x)
    near(got["dinitial_state"], dS, "dinitial_state")


def test_delta_past_two_to_the_31_elements():
    """A packed batch whose last sequence lies past element 2^31 of v, and its tiles' states past
    2^32: both directions of that sequence against 64 bits."""
    H, V, d, last = 4, 8, 128, 300
    T = 2 ** 21 + 333
    lengths = [2 ** 20, T - last - 2 ** 20, last]
    gen = torch.Generator("cuda").manual_seed(1)

    def act(heads, one):
        x = torch.empty(heads, T, d, dtype=BF16, device="cuda").normal_(generator=gen)
        if one:
            for h in range(heads):
                x[h] = unit(x[h]).to(BF16)
        return x

    q, k, v, dout = act(H, True), act(H, True), act(V, False), act(V, False)
    g = -2.0 ** -6 * torch.rand(V, T, generator=gen, device="cuda")
    b = torch.rand(V, T, generator=gen, device="cuda")
    cu = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
    scale = d ** -0.5
    out, S = gbla.delta_attention(q, k, v, g, b, final_state=True, cu_seqlens=cu)
    tail = [x[:, -last:].cpu() for x in (q, k, v, g, b, dout)]
    want, final = ref.delta(*tail[:5], scale)
    size, size_S = ref.delta_sizes(*tail[:5], scale)
    _check(out[:, -last:], want, size, c_of(last, d) + 2.0 ** -14, "out")
    _check(S[2], final, size_S.expand_as(final), c_of(last, d), "final_state")
    del out, S
    got = gbla.delta_attention_backward(q, k, v, g, b, dout, cu_seqlens=cu)
    want = ref.delta_backward(*tail, scale)
    size = ref.delta_backward_sizes(*tail, scale)
    for x, w, z in zip(("dq", "dk", "dv", "dlog_decay", "dbeta"), want, size):
        y = got[x][:, -last:]
        _check(y, w, z, c_back(last, d) + (6 * 2.0 ** -16 if y.dtype == BF16 else 0.0), x)
    del got
    torch.cuda.empty_cache()


def test_delta_step_and_norm_past_two_to_the_31_elements():
    gen = torch.Generator("cuda").manual_seed(2)
    randn = lambda *s, t=F32: torch.empty(*s, dtype=t, device="cuda").normal_(generator=gen)
    V, d, slots = 8, 128, 20001
    q, k, v = (unit(randn(2, V, d)).to(BF16) for _ in range(3))
    g, b = -randn(2, V).abs(), torch.rand(2, V, generator=gen, device="cuda")
    state = randn(slots, V, d, d)
    few = state[[slots - 1, 3]].clone()
    at = torch.tensor([slots - 1, 3], dtype=torch.int32, device="cuda")
    y = gbla.delta_step(q, k, v, g, b, state, state_indices=at)
    assert torch.equal(y, gbla.delta_step(q, k, v, g, b, few))
    assert torch.equal(state[[slots - 1, 3]], few)
    del state
    rows, width = 2 ** 21 + 5, 1024
    x, r = randn(rows, width, t=BF16), randn(rows, width, t=BF16)
    w = randn(width)
    y, s = gbla.add_rms_norm(x, w, r)
    z, t = gbla.add_rms_norm(x[-5:].clone(), w, r[-5:].clone())
    assert torch.equal(y[-5:], z) and torch.equal(s[-5:], t)
    dx = gbla.add_rms_norm_backward(s, w, x, r)["dx"]
    assert torch.equal(dx[-5:], gbla.add_rms_norm_backward(t, w, x[-5:].clone(), r[-5:].clone())["dx"])
    del x, r, y, s, dx
    torch.cuda.empty_cache()


def test_delta_on_two_streams_at_once():
    """Calls under way at the same time, each with its own scratch, give what one alone gives."""
    t = delta_case([3000, 70, 1500], True, 2, 4, 64, BF16, True, (-5, -6, -7, -8))
    args = _dev(*(t[x] for x in NAMES + ("dout",)))
    S0, dS, cu = _dev(t["S0"], t["dS"], t["cu"])
    want, Sw = gbla.delta_attention(*args[:5], initial_state=S0, final_state=True, cu_seqlens=cu)
    gw = gbla.delta_attention_backward(*args, initial_state=S0, dfinal_state=dS, cu_seqlens=cu)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs, grads = [], []
    for _ in range(4):
        for s in streams:
            outs.append(gbla.delta_attention(*args[:5], initial_state=S0, final_state=True, cu_seqlens=cu, stream=s))
            grads.append(gbla.delta_attention_backward(*args, initial_state=S0, dfinal_state=dS, cu_seqlens=cu,
                                                       stream=s))
    torch.cuda.synchronize()
    for y, S in outs:
        assert torch.equal(y, want) and torch.equal(S, Sw)
    for got in grads:
        for x in gw:
            assert torch.equal(got[x], gw[x]), x


@pytest.mark.parametrize("ragged", [False, True])
def test_delta_of_no_tokens(ragged):
    """The states pass through, whatever the scratch holds."""
    t = delta_case([0, 0], ragged, 2, 4, 32, BF16, True, (-5, -6, -7, -8))
    args = _dev(*(t[x] for x in NAMES + ("dout",)))
    S0, dS, cu = _dev(t["S0"], t["dS"], t["cu"])
    out, S = gbla.delta_attention(*args[:5], initial_state=S0, final_state=True, cu_seqlens=cu)
    assert out.shape == args[2].shape and torch.equal(S, S0)
    got = gbla.delta_attention_backward(*args, initial_state=S0, dfinal_state=dS, cu_seqlens=cu)
    assert torch.equal(got["dinitial_state"], dS) and got["dq"].shape == args[0].shape
