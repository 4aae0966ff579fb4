"""Gradients of the decay attention on the GPU where the general cases of
test_decoder_gpu.py cannot tell a small error from a rounding."""
import pytest
import torch

from paper_2606_07317_amd import gbla

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# 1 + 2^-9 + 2^-18 and 1 + 2^-9 as sums of bf16 values: their difference is 2^-18, which two
# bf16 parts of either (17 bits) do not hold and three (24 bits) do.
LONG, SHORT = [1.0, 2.0 ** -9, 2.0 ** -18], [1.0, 2.0 ** -9, 0.0]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [1, 3])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("n,s,t", [(3, 0, 1), (64, 5, 40), (200, 3, 190), (900, 10, 870)])
def test_differences_of_long_sums_are_exact(n, s, t, d, group, dtype):
    """No decay, scale 1: every product and sum here is exact in fp32, so the gradients are
    too.  The tokens lie in one tile, in different tiles, or in different units."""
    q, do = (torch.zeros(1, group, n, d, dtype=dtype, device="cuda") for _ in range(2))
    k, v = (torch.zeros(1, 1, n, d, dtype=dtype, device="cuda") for _ in range(2))
    g = torch.zeros(1, device="cuda")
    row = lambda x: torch.tensor(x, dtype=dtype, device="cuda")
    call = lambda: gbla.decay_attention_backward(q, k, v, g, do, scale=1.0)
    want = torch.zeros(d, dtype=dtype, device="cuda")
    want[:] = 2.0 ** -18
    head = group - 1

    def clear():
        for x in (q, k, v, do):
            x.zero_()

    # dv_s = (q_t k_s) do_t + (q_{t+1} k_s) do_{t+1}
    q[0, head, t, :3], q[0, head, t + 1, :3] = row(LONG), row(SHORT)
    k[0, 0, s, :3] = 1.0
    do[0, head, t], do[0, head, t + 1] = 1.0, -1.0
    assert torch.equal(call()["dv"][0, 0, s], want)
    # dk_s = (do_t v_s) q_t + (do_{t+1} v_s) q_{t+1}
    clear()
    do[0, head, t, :3], do[0, head, t + 1, :3] = row(LONG), row(SHORT)
    v[0, 0, s, :3] = 1.0
    q[0, head, t], q[0, head, t + 1] = 1.0, -1.0
    assert torch.equal(call()["dk"][0, 0, s], want)
    # dq_t = (do_t v_s) k_s + (do_t v_{s+1}) k_{s+1}
    clear()
    v[0, 0, s, :3], v[0, 0, s + 1, :3] = row(LONG), row(SHORT)
    do[0, head, t + 1, :3] = 1.0
    k[0, 0, s], k[0, 0, s + 1] = 1.0, -1.0
    assert torch.equal(call()["dq"][0, head, t + 1], want)
    # the same differences between two channels of a state's row or column, whose elements
    # three tokens make:  D = sum q do^T, dv_s = D^T k_s, dk_s = D v_s;  S = sum k v^T, dq = S do
    if t + 4 >= n:
        return
    clear()
    for i in range(3):
        q[0, head, t + i, 0], q[0, head, t + i, 1] = LONG[i], SHORT[i]
        do[0, head, t + i] = 1.0
    k[0, 0, s, 0], k[0, 0, s, 1] = 1.0, -1.0
    assert torch.equal(call()["dv"][0, 0, s], want)
    clear()
    for i in range(3):
        do[0, head, t + i, 0], do[0, head, t + i, 1] = LONG[i], SHORT[i]
        q[0, head, t + i] = 1.0
    v[0, 0, s, 0], v[0, 0, s, 1] = 1.0, -1.0
    assert torch.equal(call()["dk"][0, 0, s], want)
    clear()
    for i in range(3):
        v[0, 0, s + i, 0], v[0, 0, s + i, 1] = LONG[i], SHORT[i]
        k[0, 0, s + i] = 1.0
    do[0, head, t + 3, 0], do[0, head, t + 3, 1] = 1.0, -1.0
    assert torch.equal(call()["dq"][0, head, t + 3], want)
