"""What the GPU tests of the gated delta rule are held against can fail: the backward's bounds of
single entries stay near the gradients in long sequences and bound what errors in the inputs do,
and the checks head by head refuse gradients that are zero, negated or somebody else's."""
import pytest
import torch

from oracle import gbla_block as ref
from tests.test_decoder_gpu import BF16, F32
from tests.test_delta_accuracy_gpu import per_head
from tests.test_delta_backward_gpu import c_of
from tests.test_delta_gpu import NAMES, delta_case

GRADS = ("dq", "dk", "dv", "dlog_decay", "dbeta", "dinitial_state")


def _case(n, d, dtype, states=True, rates=(-5, -8)):
    t = delta_case([n], False, 1, len(rates), d, dtype, states, rates)
    args = [t[x][0] for x in NAMES + ("dout",)]
    return args, (t["S0"][0], t["dS"][0]) if states else (None, None)


@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_backwards_bounds_do_not_grow_with_the_sequence(d, states):
    """Sixteen times the tokens: sums over the sequence (dlog_decay's) are sixteen times as large and
    the states, of horizons of hundreds of tokens, four times each, 256 in all; a bound that fed
    itself would grow by powers.  Those of dq, dv, dbeta and dinitial_state are within a small multiple of them at
    any length; dk and dlog_decay, whose bounds add up products of columns' lengths, are held by
    the norms of their heads."""
    ratio = {}
    for n in (64, 1000):
        args, (S0, dS) = _case(n, d, F32, states)
        want = ref.delta_backward(*args, d ** -0.5, S0, dS)
        size = ref.delta_backward_sizes(*args, d ** -0.5, S0, dS)
        ratio[n] = {x: (c_of(n, d) * z.double().median() / w.square().mean().sqrt()).item()
                    for x, w, z in zip(GRADS, want, size)}
    for x in GRADS:
        assert ratio[1000][x] <= 256 * ratio[64][x], (x, ratio)
    for x in ("dq", "dv", "dbeta", "dinitial_state"):
        assert ratio[1000][x] <= 16, (x, ratio)


@pytest.mark.parametrize("which", ["v", "dout", "S0", "dS"])
def test_backwards_bounds_hold_of_a_perturbed_run(which):
    """Values off by a relative 1e-3 move gradients by no more than 1e-3 of the bounds (their
    derivation is linear; 1 % for the products of two errors)."""
    args, states = _case(200, 8 * 4, F32)
    base = ref.delta_backward(*args, 0.5, *states)
    size = ref.delta_backward_sizes(*args, 0.5, *states)
    off = lambda x: x.double() * (1 + 1e-3 * torch.sign(torch.randn(x.shape, generator=torch.Generator().manual_seed(3))))
    args, states = list(args), list(states)
    if which in ("S0", "dS"):
        states[which == "dS"] = off(states[which == "dS"])
    else:
        i = (NAMES + ("dout",)).index(which)
        args[i] = off(args[i])
    for x, a, b, z in zip(GRADS, ref.delta_backward(*args, 0.5, *states), base, size):
        assert ((a - b).abs() <= 1.01e-3 * z + 1e-12).all(), x


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 128)])
def test_wrong_gradients_are_refused(dtype, d):
    """Zero, negated, another head's, another token's, one entry in another's place."""
    args, (S0, dS) = _case(300, d, dtype)
    for name, want in zip(GRADS, ref.delta_backward(*args, d ** -0.5, S0, dS)):
        kind = dtype if name in ("dq", "dk", "dv") else F32
        want = want.repeat(2, *[1] * (want.dim() - 1)) if want.shape[0] == 1 else want
        per_head(want.to(kind), want, name)
        moved = want.clone()
        moved[0] = moved[0].roll(1, 0)
        one = want.clone().flatten(1)
        one[1, 7] = one[1, 7] + one[1].square().mean().sqrt()
        half = want.clone()
        half[1] = 0
        wrong = [torch.zeros_like(want), -want, half, moved, one.view_as(want)]
        if want.shape[0] == 2 and not torch.equal(want[0], want[1]):
            wrong.append(want.flip(0))
        for bad in wrong:
            with pytest.raises(AssertionError):
                per_head(bad.to(kind), want, name)


@pytest.mark.parametrize("parts,ok", [(1, False), (3, True)])
def test_states_of_too_few_parts_are_refused(parts, ok):
    """The recurrence with u cut to bf16 parts before it enters the state, as a tile's products are."""
    n, d = 300, 64
    (q, k, v, g, b, _), (S0, _) = _case(n, d, BF16)
    _, want = ref.delta(q, k, v, g, b, d ** -0.5, S0)
    S = S0.double()
    for t in range(n):
        S = torch.exp(g[:, t, None, None].double()) * S
        u = b[:, t, None] * (v[:, t].double() - torch.matmul(k[:, t, None, :].double(), S)[:, 0])
        kept = torch.zeros_like(u)
        for _ in range(parts):
            kept = kept + (u - kept).to(BF16).double()
        S = S + k[:, t, :, None].double() * kept[:, None, :]
    if ok:
        per_head(S.float(), want, "state")
    else:
        with pytest.raises(AssertionError):
            per_head(S.float(), want, "state")
