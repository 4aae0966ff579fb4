"""The decoder's operators at the sizes of long prompts and large batches: the longer units of
the decay attention, sequences of more units than one round of their scan takes, tensors past
2^31 elements, many query heads to a key head; and the gradient of the decay against bounds
that it could miss.

Tolerances are those of test_decoder_gpu.py (``_c``, in bf16 without the forward's 2^-16 for
gradients, whose products have fp32's accuracy for both types).
"""
import pytest
import torch

from oracle import gbla_decoder as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, U, _c, _check, _decay_case, _dev, _gen, _pair_size, _pieces, _randn

pytestmark = pytest.mark.gpu


def _compare(t, got_out, got_S, got, lengths, ragged, dtype, heads, seqs):
    """Forward and backward results of key heads ``heads`` in sequences ``seqs`` against the
    recurrence; the decay's gradient too where ``seqs`` is the whole batch."""
    H, K = t["q"].shape[-3], t["k"].shape[-3]
    G, d = H // K, t["q"].shape[-1]
    scale = d ** -0.5
    qs = [h * G + j for h in heads for j in range(G)]
    g = t["g"][heads]
    total, bound = torch.zeros(len(heads)).double(), torch.zeros(len(heads)).double()
    parts = {n: list(_pieces(x, lengths, ragged)) for n, x in
             [(n, t[n]) for n in ("q", "k", "v", "dout")] + [("out", got_out)] + [(n, got[n]) for n in ("dq", "dk", "dv")]}
    for s in seqs:
        q, do = parts["q"][s][qs].cpu(), parts["dout"][s][qs].cpu()
        k, v = parts["k"][s][heads].cpu(), parts["v"][s][heads].cpu()
        S0 = t["S0"][s][heads] if t["S0"] is not None else None
        dS = t["dS"][s][heads] if t["dS"] is not None else None
        n = lengths[s]
        c = (2 * d + 144 + n / 64) * 2 * U
        want, final = ref.decay(q, k, v, g, scale, S0)
        size, size_S = ref.decay_sizes(q, k, v, g, scale, S0)
        _check(parts["out"][s][qs], want, size, _c(n, d, dtype), "out")
        _check(got_S[s][heads], final, size_S, c, "final_state")
        want = ref.decay_backward(q, k, v, g, do, scale, S0, dS)
        size = ref.decay_backward_sizes(q, k, v, g, do, scale, S0, dS)
        for i, (name, which) in enumerate((("dq", qs), ("dk", heads), ("dv", heads))):
            _check(parts[name][s][which], want[i], size[i], c, name)
        if S0 is not None:
            _check(got["dinitial_state"][s][heads], want[4], size[4], c, "dinitial_state")
        total += want[3]
        bound += c * size[3]
    if len(seqs) == len(lengths):
        _check(got["dlog_decay"][heads], total, bound, 1.0, "dlog_decay")


def _run(t, max_seqlen=None):
    args = _dev(t["q"], t["k"], t["v"], t["g"])
    do, S0, dS, cu = _dev(t["dout"], t["S0"], t["dS"], t["cu"])
    out, S = gbla.decay_attention(*args, initial_state=S0, final_state=True, cu_seqlens=cu, max_seqlen=max_seqlen)
    got = gbla.decay_attention_backward(*args, do, initial_state=S0, dfinal_state=dS, cu_seqlens=cu,
                                        max_seqlen=max_seqlen)
    return out, S, got


# lengths, ragged, H, K, d, dtype, states, log decays; key heads and sequences compared
LONG = [
    # units of 128 tokens, more than one round (32 units) of the scan, and than two
    (([4300], False, 1, 1, 32, BF16, True, [-0.002]), [0], [0]),
    (([4300], False, 2, 1, 32, F32, False, [-0.0005]), [0], [0]),
    (([70, 8500, 0, 4097], True, 1, 1, 32, BF16, True, [-0.001]), [0], [0, 1, 2, 3]),
    (([4200, 129], True, 1, 1, 64, F32, True, [-0.003]), [0], [0, 1]),
    (([4230], False, 1, 1, 128, BF16, True, [-0.001]), [0], [0]),
    # units of 256
    (([4200], False, 32, 32, 32, BF16, True, [-0.0005 * (i + 1) for i in range(32)]), [0, 31], [0]),
    # units of 512: split, with more than one round, and walked whole
    (([4200], False, 64, 64, 32, F32, False, [-0.0005 * (i + 1) for i in range(64)]), [0, 63], [0]),
    (([17000], False, 16, 16, 32, BF16, True, [-0.0002 * (i + 1) for i in range(16)]), [1], [0]),
    (([4100], False, 128, 64, 64, BF16, True, [-0.0005 * (i + 1) for i in range(64)]), [40], [0]),
    (([1500] * 16, False, 16, 16, 32, F32, True, [-0.001 * (i + 1) for i in range(16)]), [3], [0, 15]),
    (([1100] * 16, False, 16, 16, 64, BF16, True, [-0.001 * (i + 1) for i in range(16)]), [15], [15]),
    # query heads that share, at every d and type
    (([200], False, 3, 1, 32, F32, True, [-0.01]), [0], [0]),
    (([330], False, 4, 1, 64, BF16, True, [-0.01]), [0], [0]),
    (([330], False, 6, 2, 64, F32, True, [-0.01, -0.002]), [0, 1], [0]),
    (([300], False, 8, 2, 128, BF16, True, [-0.01, -0.002]), [0, 1], [0]),
    (([700, 40, 130], True, 3, 1, 128, F32, True, [-0.01]), [0], [0, 1, 2]),
    (([260], False, 8, 2, 128, F32, True, [-0.01, -0.002]), [0, 1], [0]),
]


@pytest.mark.parametrize("case,heads,seqs", LONG, ids=lambda x: None if not isinstance(x, tuple) else
                         "%d-%s" % (max(x[0]), "-".join(map(str, x[2:7]))))
def test_long_sequences_and_long_units(case, heads, seqs):
    t = _decay_case(*case)
    _compare(t, *_run(t, max(case[0])), case[0], case[1], case[5], heads, seqs)


# ---------------------------------------------------------------------------
# The gradient of the decay, where all its terms have one sign.
# ---------------------------------------------------------------------------
SIGNED = [
    (([2], False, 1, 1, 32, F32, False, [-0.01])),
    (([64], False, 2, 1, 64, BF16, False, [-0.005])),
    (([64], False, 2, 2, 64, F32, True, [-0.005, -0.05])),
    (([200] * 2, False, 2, 2, 32, BF16, True, [-0.001, -0.02])),
    (([150], False, 4, 2, 128, BF16, True, [-0.004, -0.03])),
    (([150], False, 2, 1, 128, F32, True, [-0.004])),
    (([700], False, 2, 2, 64, BF16, True, [-0.002, -0.01])),      # units
    (([640], False, 2, 1, 128, BF16, False, [-0.003])),
    (([777], False, 2, 2, 64, F32, False, [-0.002, -0.01])),
    (([1300], False, 3, 1, 32, F32, True, [-0.001])),
    (([700, 0, 1, 128, 513], True, 2, 1, 64, BF16, True, [-0.005])),
    (([30, 900, 64], True, 2, 2, 128, F32, True, [-0.003, -0.01])),
    (([4300], False, 1, 1, 32, BF16, True, [-0.0005])),           # rounds of units
    (([4200], False, 64, 64, 32, BF16, True, [-0.002] * 64)),     # units of 512
    (([1500] * 16, False, 16, 16, 32, BF16, True, [-0.002] * 16)),
]


@pytest.mark.parametrize("case,only", [(c, o) for c in SIGNED for o in ("all", "initial", "final", "neither")
                                       if c[6] or o == "all"],  # with which states
                         ids=lambda x: x if isinstance(x, str) else "%d-%s" % (max(x[0]), "-".join(map(str, x[1:7]))))
def test_gradient_of_the_decay(case, only):
    """Positive inputs, so that the gradient is the sum of its terms' sizes and the bound a
    small part of it: a part left out, counted twice or of the wrong sign fails."""
    lengths, ragged, H, K, d, dtype, states, g = case
    t = _decay_case(*case)
    for n in ("q", "k", "v", "dout"):
        t[n] = t[n].abs()
    for n in ("S0", "dS"):
        t[n] = t[n].abs() if t[n] is not None and only in ("all", {"S0": "initial", "dS": "final"}[n]) else None
    args = _dev(t["q"], t["k"], t["v"], t["g"], t["dout"])
    S0, dS, cu = _dev(t["S0"], t["dS"], t["cu"])
    got = gbla.decay_attention_backward(*args, initial_state=S0, dfinal_state=dS, cu_seqlens=cu,
                                        max_seqlen=max(lengths))["dlog_decay"]
    scale, G = d ** -0.5, H // K
    heads = [0, K - 1] if K > 2 else list(range(K))
    want, bound = torch.zeros(len(heads)).double(), torch.zeros(len(heads)).double()
    qs = [h * G + j for h in heads for j in range(G)]
    for s, (q, k, v, do) in enumerate(zip(*(_pieces(t[n], lengths, ragged) for n in ("q", "k", "v", "dout")))):
        state = lambda n: t[n][s][heads] if t[n] is not None else None
        args = (q[qs], k[heads], v[heads], t["g"][heads], do[qs], scale, state("S0"), state("dS"))
        want += ref.decay_backward(*args)[3]
        bound += (2 * d + 144 + lengths[s] / 64) * 2 * U * ref.decay_backward_sizes(*args)[3]
    assert (bound < 0.05 * want).all()
    _check(got[heads], want, bound, 1.0, "dlog_decay")


# ---------------------------------------------------------------------------
# Past 2^31 elements
# ---------------------------------------------------------------------------
B31, H31, N31, D31 = 2100, 16, 512, 128  # 2.2e9 elements


def _need(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip("needs %d GB of free memory" % gigabytes)


def _large(seed, ragged):
    torch.manual_seed(seed)
    shape = (H31, B31 * N31, D31) if ragged else (B31, H31, N31, D31)
    return torch.empty(shape, dtype=BF16, device="cuda").normal_()


@pytest.mark.parametrize("ragged", [False, True])
def test_decay_backward_beyond_32_bit_offsets(ragged):
    """The first and the last sequence and head of a batch of more than 2^31 elements."""
    _need(60)
    x, do = _large(0, ragged), _large(1, ragged)
    g = torch.linspace(-0.05, -0.001, H31)
    cu = (torch.arange(B31 + 1) * N31).to(torch.int32) if ragged else None
    how = dict(cu_seqlens=_dev(cu)[0], max_seqlen=N31 if ragged else None)
    out, S = gbla.decay_attention(x, x, x, g.cuda(), final_state=True, **how)
    got = gbla.decay_attention_backward(x, x, x, g.cuda(), do, **how)
    for s, h in ((0, 0), (B31 - 1, H31 - 1), (B31 - 1, 0), (B31 // 2, H31 - 1)):
        piece = lambda y: (y[h, s * N31:(s + 1) * N31] if ragged else y[s, h])[None]
        a, b, scale = piece(x).cpu(), piece(do).cpu(), D31 ** -0.5
        want, final = ref.decay(a, a, a, g[h:h + 1], scale)
        size, size_S = ref.decay_sizes(a, a, a, g[h:h + 1], scale)
        c = (2 * D31 + 144 + N31 / 64) * 2 * U
        _check(piece(out), want, size, _c(N31, D31, BF16), "out")
        _check(S[s, h][None], final, size_S, c, "final_state")
        want = ref.decay_backward(a, a, a, g[h:h + 1], b, scale)
        size = ref.decay_backward_sizes(a, a, a, g[h:h + 1], b, scale)
        for i, n in enumerate(("dq", "dk", "dv")):
            _check(piece(got[n]), want[i], size[i], c, n)
    del out, S
    # the decay's gradient: the same units' parts, added in 64 bits, and a rounding for each call
    parts, sizes, at = torch.zeros(H31).double(), torch.zeros(H31).double(), 0
    for n in (700, 700, 700):
        sub = (lambda y: y[:, at * N31:(at + n) * N31].contiguous()) if ragged else (lambda y: y[at:at + n].contiguous())
        cu = (torch.arange(n + 1) * N31).to(torch.int32).cuda() if ragged else None
        y = sub(x)
        part = gbla.decay_attention_backward(y, y, y, g.cuda(), sub(do), cu_seqlens=cu,
                                             max_seqlen=N31 if ragged else None)["dlog_decay"].cpu().double()
        parts, sizes, at = parts + part, sizes + part.abs(), at + n
    assert ((got["dlog_decay"].cpu().double() - parts).abs() <= 2 * U * sizes).all()


@pytest.mark.parametrize("ragged", [False, True])
def test_rope_beyond_32_bit_offsets(ragged):
    _need(60)
    x, dy = _large(2, ragged), _large(3, ragged)
    w = 1 + 0.3 * _randn(_gen(0), H31, D31)
    cu = (torch.arange(B31 + 1) * N31).to(torch.int32) if ragged else None
    how = dict(cu_seqlens=_dev(cu)[0])
    q, k = gbla.qk_norm_rope(x, x, w.cuda(), w.cuda(), **how)
    assert torch.equal(q, k)
    del k
    got = gbla.qk_norm_rope_backward(x, x, w.cuda(), w.cuda(), dy, dy, **how)
    pos = torch.arange(N31)
    for s, h in ((0, 0), (B31 - 1, H31 - 1), (B31 - 1, 0), (B31 // 2, H31 - 1)):
        piece = lambda y: (y[h, s * N31:(s + 1) * N31] if ragged else y[s, h])[None]
        a, wh = piece(x).cpu(), w[h:h + 1]
        _check(piece(q), ref.rope(a, wh, pos, D31), _pair_size(ref.rope(a, wh, pos, 0), D31, False),
               (D31 / 8 + 24) * 2 * U, "q")
        b = piece(dy).cpu()
        want, _ = ref.rope_backward(a, wh, pos, b, D31)
        r = 1 / torch.sqrt((a.double() ** 2).mean(-1, keepdim=True) + 1e-6)
        xn, uw = (a.double() * r).abs(), _pair_size(b.double(), D31, False) * wh.double()[:, None, :].abs()
        size = r * (uw + xn * (uw * xn).mean(-1, keepdim=True))
        _check(piece(got["dq"]), want, size, (D31 / 8 + 40) * 2 * U, "dq")
    assert torch.equal(got["dq"], got["dk"]) and torch.equal(got["dq_w"], got["dk_w"])
    del q
    # the weights' gradient: of the batch's parts.  A sum of n terms of size 1 (in the mean of
    # their squares, so at most 1.1 n in all), 32 of whose additions round before the
    # compensated ones, on both sides.
    parts, at = torch.zeros(H31, D31).double(), 0
    for n in (700, 700, 700):
        sub = (lambda y: y[:, at * N31:(at + n) * N31].contiguous()) if ragged else (lambda y: y[at:at + n].contiguous())
        cu = (torch.arange(n + 1) * N31).to(torch.int32).cuda() if ragged else None
        y, z = sub(x), sub(dy)
        parts += gbla.qk_norm_rope_backward(y, y, w.cuda(), w.cuda(), z, z, cu_seqlens=cu)["dq_w"].cpu().double()
        at += n
    over = (got["dq_w"].cpu().double() - parts).abs().max()
    assert over <= 64 * U * 1.1 * B31 * N31 and parts.abs().max() > 100 * 64 * U * 1.1 * B31 * N31


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_step_beyond_32_bit_offsets(dtype):
    """States of more than 2^31 elements."""
    slots, K, H, d = 17000, 8, 16, 128
    _need(20)
    torch.manual_seed(4)
    state = torch.empty(slots, K, d, d, device="cuda").normal_()
    gen = _gen(5)
    q, k, v = (_randn(gen, 4, h, d, dtype=dtype) for h in (H, K, K))
    g = -torch.rand(K, generator=gen)
    rows = [slots - 1, 0, slots - 2, slots // 2]
    before = [state[s].cpu() for s in rows]
    near = state[slots - 3].clone()
    out = gbla.decay_step(*_dev(q, k, v, g), state, state_indices=torch.tensor(rows, dtype=torch.int32).cuda())
    for n, s in enumerate(rows):
        args = (q[n][:, None], k[n][:, None], v[n][:, None], g, d ** -0.5, before[n])
        want, final = ref.decay(*args)
        size, size_S = ref.decay_sizes(*args)
        _check(out[n], want[:, 0], size[:, 0], (d + 8) * 2 * U, "out")
        _check(state[s], final, size_S, 8 * U, "state")
    assert torch.equal(near, state[slots - 3])


def test_prompt_into_slots_and_a_step_from_them():
    """A prompt's final states written into neighbouring slots of a pool, which a step names."""
    gen = _gen(6)
    B, H, K, d, n = 3, 4, 2, 64, 150
    q, k, v = (_randn(gen, B, h, n + 1, d, dtype=BF16) for h in (H, K, K))
    g = torch.tensor([-0.01, -0.1])
    pool = torch.full((8, K, d, d), 3.0, device="cuda")
    cut = lambda x: x[:, :, :n].contiguous().cuda()
    _, S = gbla.decay_attention(cut(q), cut(k), cut(v), g.cuda(), final_state=pool[2:5])
    last = lambda x: x[:, :, n].contiguous().cuda()
    out = gbla.decay_step(last(q), last(k), last(v), g.cuda(), pool,
                          state_indices=torch.tensor([2, 3, 4], dtype=torch.int32).cuda())
    assert S.data_ptr() == pool[2:5].data_ptr() and (pool[[0, 1, 5, 6, 7]] == 3.0).all()
    for b in range(B):
        want, final = ref.decay(q[b], k[b], v[b], g, d ** -0.5)
        size, size_S = ref.decay_sizes(q[b], k[b], v[b], g, d ** -0.5)
        c = (2 * d + 144 + n / 64 + 8) * 2 * U
        _check(out[b], want[:, n], size[:, n], c, "out")
        _check(pool[2 + b], final, size_S, c, "state")
