"""Infinite and NaN values in the decoder's operators: they reach the results that they
have a part in, and no others."""
import pytest
import torch

from oracle import gbla_decoder as ref
from paper_2606_07317_amd import gbla

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("bad", [INF, NAN])
@pytest.mark.parametrize("flags", [0, gbla.ROPE_PAIRS])
@pytest.mark.parametrize("d,rotary", [(32, 8), (64, 0), (128, 96)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_channels_that_do_not_rotate_stay(dtype, d, rotary, flags, bad):
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(2, 3, 40, d, generator=gen).to(dtype).cuda()
    flags |= gbla.NO_NORM
    for ch in (rotary, d - 1):
        y = x.clone()
        y[..., ch] = bad
        others = [c for c in range(rotary, d) if c != ch]
        for out in (gbla.qk_norm_rope(y, y, None, None, rotary_dim=rotary, flags=flags),
                    [gbla.qk_norm_rope_backward(x, x, None, None, y, y, rotary_dim=rotary, flags=flags)[n]
                     for n in ("dq", "dk")]):
            for z in out:
                assert torch.equal(z[..., others], x[..., others])
                assert not torch.isfinite(z[..., ch]).any()
                assert torch.isfinite(z[..., :rotary]).all()


@pytest.mark.parametrize("flags", [0, gbla.ROPE_PAIRS])
def test_the_norm_of_an_infinite_channel_leaves_zeros(flags):
    """x / sqrt(inf) is 0 in every finite channel."""
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(1, 2, 9, 64, generator=gen).cuda()
    x[..., 63] = INF
    w = torch.ones(2, 64, device="cuda")
    for z in gbla.qk_norm_rope(x, x, w, w, rotary_dim=32, flags=flags):
        assert (z[..., :63] == 0).all()


# ---------------------------------------------------------------------------
# Decay attention: the results are finite exactly where the recurrence's are.
# ---------------------------------------------------------------------------
U = 2.0 ** -24
# lengths, ragged, H, K, d, dtype
DECAY = [
    ([130], False, 1, 1, 32, BF16),
    ([200], False, 4, 2, 64, BF16),
    ([150], False, 2, 1, 128, BF16),
    ([150], False, 2, 2, 128, BF16),
    ([130], False, 2, 2, 32, F32),
    ([100], False, 3, 1, 64, F32),
    ([140], False, 2, 2, 128, F32),
    ([700], False, 2, 2, 64, BF16),            # several units
    ([70, 0, 650, 40], True, 2, 1, 32, BF16),
    ([20, 130], True, 2, 2, 64, F32),
]
_IDS = ["%s-%d-%s" % ("-".join(map(str, c[0])), c[4], "-".join(map(str, c[2:4]))) + str(c[5])[5:] for c in DECAY]


def _case(lengths, ragged, H, K, d, dtype):
    gen = torch.Generator().manual_seed(1)
    T, B, n = sum(lengths), len(lengths), lengths[0]
    act = (lambda h: (h, T, d)) if ragged else (lambda h: (B, h, n, d))
    t = {x: torch.randn(*act(h), generator=gen).to(dtype) for x, h in (("q", H), ("k", K), ("v", K), ("dout", H))}
    t["g"] = -0.02 * (1 + torch.arange(K, dtype=F32))
    for x in ("S0", "dS"):
        t[x] = torch.randn(B, K, d, d, generator=gen)
    t["cu"] = torch.tensor([0] + lengths).cumsum(0).to(torch.int32) if ragged else None
    return t


def _pieces(x, lengths, ragged):
    at = 0
    for s, n in enumerate(lengths):
        yield x[:, at:at + n] if ragged else x[s]
        at += n


def _same_places(got, want, clean, size, c, name):
    """Finite where ``want`` is, and there within half a step and c * size of the results
    ``clean`` of inputs without the bad values."""
    got = got.cpu()
    step = torch.finfo(got.dtype).eps / 2
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), "%s: %d finite that should not be, %d not finite that should" % (
        name, (torch.isfinite(got) & ~fine).sum(), (~torch.isfinite(got) & fine).sum())
    over = (got.double() - clean).abs() - (step * clean.abs() * (1 + 2 * step) + c * size + 1e-37)
    assert (over[fine] <= 0).all(), name


def _bad(t, lengths, ragged, where, value):
    """Copies of the tensors with ``value`` and with 0 in one channel of one head of each named
    tensor, at these tokens (counted over the batch)."""
    with_bad, clean = dict(t), dict(t)
    for name, token, channel in where:
        for out, x in ((with_bad, value), (clean, 0.0)):
            y = out[name].clone()
            if name in ("S0", "dS"):
                y[token, -1, channel, channel + 1] = x
            elif ragged:
                y[-1, token, channel] = x
            else:
                y[0, -1, token, channel] = x
            out[name] = y
    return with_bad, clean


@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("where", [
    [("v", 20, 5)], [("k", 20, 5)], [("q", 20, 5)], [("v", 63, 0), ("k", 64, 31)], [("S0", 0, 7)],
    [("k", 99, 3), ("v", 99, 4)]], ids=lambda w: "-".join("%s%d" % x[:2] for x in w))
@pytest.mark.parametrize("case", DECAY, ids=_IDS)
def test_decay_forward_is_finite_where_the_recurrence_is(case, where, value):
    lengths, ragged, H, K, d, dtype = case
    t, clean = _bad(_case(*case), lengths, ragged, where, value)
    dev = lambda x: None if x is None else x.cuda()
    out, S = gbla.decay_attention(*map(dev, (t["q"], t["k"], t["v"], t["g"])), initial_state=dev(t["S0"]),
                                  final_state=True, cu_seqlens=dev(t["cu"]))
    parts = [list(_pieces(x, lengths, ragged)) for x in (t["q"], t["k"], t["v"], clean["q"], clean["k"], clean["v"], out)]
    for s, (q, k, v, q0, k0, v0, y) in enumerate(zip(*parts)):
        scale = d ** -0.5
        want = ref.decay(q, k, v, t["g"], scale, t["S0"][s])
        plain = ref.decay(q0, k0, v0, t["g"], scale, clean["S0"][s])
        size = ref.decay_sizes(q0, k0, v0, t["g"], scale, clean["S0"][s])
        c = (2 * d + 144 + lengths[s] / 64) * 2 * U
        _same_places(y, want[0], plain[0], size[0], c + (2.0 ** -16 if dtype == BF16 else 0.0), "out")
        _same_places(S[s], want[1], plain[1], size[1], c, "final_state")


@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("where", [
    [("v", 20, 5)], [("k", 20, 5)], [("q", 20, 5)], [("dout", 20, 5)], [("q", 63, 0), ("dout", 64, 31)],
    [("S0", 0, 7)], [("dS", 0, 7)], [("q", 99, 3), ("k", 98, 4)]],
    ids=lambda w: "-".join("%s%d" % x[:2] for x in w))
@pytest.mark.parametrize("case", DECAY, ids=_IDS)
def test_decay_backward_is_finite_where_the_recurrence_is(case, where, value):
    lengths, ragged, H, K, d, dtype = case
    t, clean = _bad(_case(*case), lengths, ragged, where, value)
    dev = lambda x: None if x is None else x.cuda()
    got = gbla.decay_attention_backward(*map(dev, (t["q"], t["k"], t["v"], t["g"], t["dout"])),
                                        initial_state=dev(t["S0"]), dfinal_state=dev(t["dS"]), cu_seqlens=dev(t["cu"]))
    names = ("q", "k", "v", "dout")
    parts = [list(_pieces(x, lengths, ragged)) for x in
             [t[n] for n in names] + [clean[n] for n in names] + [got[n] for n in ("dq", "dk", "dv")]]
    for s, (q, k, v, do, q0, k0, v0, do0, dq, dk, dv) in enumerate(zip(*parts)):
        scale = d ** -0.5
        want = ref.decay_backward(q, k, v, t["g"], do, scale, t["S0"][s], t["dS"][s])
        plain = ref.decay_backward(q0, k0, v0, t["g"], do0, scale, clean["S0"][s], clean["dS"][s])
        size = ref.decay_backward_sizes(q0, k0, v0, t["g"], do0, scale, clean["S0"][s], clean["dS"][s])
        c = (2 * d + 144 + lengths[s] / 64) * 2 * U
        for i, (name, y) in enumerate((("dq", dq), ("dk", dk), ("dv", dv))):
            _same_places(y, want[i], plain[i], size[i], c, name)
        _same_places(got["dinitial_state"][s], want[4], plain[4], size[4], c, "dinitial_state")


@pytest.mark.parametrize("dtype,n", [(BF16, 600), (F32, 130)])
def test_decay_backward_in_place_where_rows_are_formed_again(dtype, n):
    """dinitial_state in dfinal_state's buffer, whose old values the second pass needs."""
    t = _case([n], False, 2, 2, 64, dtype)
    t["q"][0, 0, 30, 3] = INF
    args = [t[x].cuda() for x in ("q", "k", "v", "g", "dout")]
    S0, dS = t["S0"].cuda(), t["dS"].cuda()
    a = gbla.decay_attention_backward(*args, initial_state=S0, dfinal_state=dS)
    b = gbla.decay_attention_backward(*args, initial_state=S0, dfinal_state=dS, grads=dict(dinitial_state=dS))
    for name in a:
        assert torch.equal(torch.nan_to_num(a[name]), torch.nan_to_num(b[name])), name


# ---------------------------------------------------------------------------
# A decay of 0: tokens and states have no part in anything after them.
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("value", [None, INF, NAN])
@pytest.mark.parametrize("g", [-INF, -200.0])
@pytest.mark.parametrize("case", DECAY, ids=_IDS)
def test_decay_of_zero_forgets(case, g, value):
    """One head without memory (the last) beside ones with: its results are each token's own."""
    lengths, ragged, H, K, d, dtype = case
    where = [("v", 20, 5), ("k", 21, 6), ("q", 22, 7), ("dout", 23, 8), ("S0", 0, 3), ("dS", 0, 9)]
    t = _case(*case)
    t, clean = _bad(t, lengths, ragged, where, value) if value is not None else (t, t)
    log_decay = t["g"].clone()
    log_decay[-1] = g
    dev = lambda x: None if x is None else x.cuda()
    args = [dev(x) for x in (t["q"], t["k"], t["v"], log_decay)]
    how = dict(initial_state=dev(t["S0"]), cu_seqlens=dev(t["cu"]))
    out, S = gbla.decay_attention(*args, final_state=True, **how)
    got = gbla.decay_attention_backward(*args, dev(t["dout"]), dfinal_state=dev(t["dS"]), **how)
    scale, G = d ** -0.5, H // K
    outs = [_pieces(x, lengths, ragged) for x in (t["q"], t["k"], t["v"], t["dout"], out, got["dq"], got["dk"], got["dv"])]
    cleans = [_pieces(clean[n], lengths, ragged) for n in ("q", "k", "v", "dout")]
    for s, ((q, k, v, do, y, dq, dk, dv), z) in enumerate(zip(zip(*outs), zip(*cleans))):
        def own(q, k, v, do, dS, S0):
            q, do, k, v = q[-G:].double(), do[-G:].double(), k[-1].double(), v[-1].double()
            a, b = scale * (q * k).sum(-1, keepdim=True), scale * (do * v).sum(-1, keepdim=True)
            gk, gv = (b * q).sum(0), (a * do).sum(0)
            if len(k):
                gk[-1] += dS.double() @ v[-1]
                gv[-1] += dS.double().T @ k[-1]
            final = k[-1][:, None] * v[-1] if len(k) else S0.double()
            return a * v, b * k, gk, gv, final, torch.zeros(d, d).double() if len(k) else dS.double()
        want = own(q, k, v, do, t["dS"][s, -1], t["S0"][s, -1])
        plain = own(*z, clean["dS"][s, -1], clean["S0"][s, -1])
        size = own(*(x.abs() for x in z), clean["dS"][s, -1].abs(), clean["S0"][s, -1].abs())
        c = (2 * d + 144) * 2 * U
        for i, (name, x) in enumerate((("out", y[-G:]), ("dq", dq[-G:]), ("dk", dk[-1]), ("dv", dv[-1]),
                                       ("final_state", S[s, -1]), ("dinitial_state", got["dinitial_state"][s, -1]))):
            _same_places(x, want[i], plain[i], size[i], c, name)
    assert got["dlog_decay"][-1] == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("g", [-INF, -200.0])
def test_step_with_a_decay_of_zero_forgets(g, d, dtype):
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(3, h, d, generator=gen).to(dtype) for h in (4, 2, 2))
    state = torch.randn(2, 2, d, d, generator=gen)
    state[1] = INF
    state[0, 1, 2] = NAN
    S = state.cuda()
    out = gbla.decay_step(q.cuda(), k.cuda(), v.cuda(), torch.tensor([g, g]).cuda(), S,
                          state_indices=torch.tensor([1, 0, 1], dtype=torch.int32).cuda())
    x = (q.double().view(3, 2, 2, d) * k.double()[:, :, None]).sum(-1, keepdim=True) * d ** -0.5
    want = (x * v.double()[:, :, None]).view(3, 4, d)
    size = ((q.double().view(3, 2, 2, d) * k.double()[:, :, None]).abs().sum(-1, keepdim=True)
            * d ** -0.5 * v.double()[:, :, None].abs()).view(3, 4, d)
    _same_places(out, want, want, size, (d + 8) * 2 * U, "out")
    for slot, n in ((0, 1), (1, 2)):
        final = k[n].double()[:, :, None] * v[n].double()[:, None]
        _same_places(S[slot], final, final, final.abs(), 8 * U, "state")


@pytest.mark.parametrize("where", [[("q", 20, 5)], [("dout", 20, 5)], [("dS", 0, 7)]], ids=lambda w: w[0][0])
@pytest.mark.parametrize("case", DECAY, ids=_IDS)
def test_decay_backward_without_the_decay_gradient_is_the_same(case, where):
    """What calls for the second pass does not depend on whether the decay's gradient is wanted."""
    t, _ = _bad(_case(*case), case[0], case[1], where, NAN)
    dev = lambda x: None if x is None else x.cuda()
    args = [dev(t[x]) for x in ("q", "k", "v", "g", "dout")]
    how = dict(initial_state=dev(t["S0"]), dfinal_state=dev(t["dS"]), cu_seqlens=dev(t["cu"]))
    a = gbla.decay_attention_backward(*args, **how)
    b = gbla.decay_attention_backward(*args, decay_grad=False, **how)
    for n in b:
        assert torch.equal(torch.isnan(a[n]), torch.isnan(b[n])) and torch.equal(
            torch.nan_to_num(a[n]), torch.nan_to_num(b[n])), n
