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
from tests.test_delta_gpu import NAMES, delta_case, own, pieces_of

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
