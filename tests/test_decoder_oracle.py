"""The 64-bit references of the decoder's operators against other forms of the same
mathematics: sums over all earlier tokens, complex rotations, central differences."""
import pytest
import torch

from oracle import gbla_decoder as ref


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("H,K,n,d", [(1, 1, 1, 4), (2, 1, 7, 4), (4, 2, 19, 8)])
def test_recurrence_is_the_sum_over_earlier_tokens(H, K, n, d):
    q, k, v, S0 = _randn(0, H, n, d), _randn(1, K, n, d), _randn(2, K, n, d), _randn(3, K, d, d)
    g = -_randn(4, K).abs()
    out, S = ref.decay(q, k, v, g, 0.5, S0)
    i = torch.arange(n).double()
    for h in range(H):
        j = h * K // H
        w = torch.exp(g[j] * (i[:, None] - i[None, :])) * (i[:, None] >= i[None, :])
        y = (q[h] @ k[j].T * w) @ v[j] + torch.exp(g[j] * (i + 1))[:, None] * (q[h] @ S0[j])
        assert torch.allclose(out[h], 0.5 * y, rtol=1e-12, atol=1e-12)
    for j in range(K):
        y = torch.exp(g[j] * n) * S0[j] + (torch.exp(g[j] * (n - 1 - i))[:, None] * k[j]).T @ v[j]
        assert torch.allclose(S[j], y, rtol=1e-12, atol=1e-12)


def test_recurrence_continues_from_its_own_state():
    q, k, v, g = _randn(0, 2, 11, 4), _randn(1, 1, 11, 4), _randn(2, 1, 11, 4), torch.tensor([-0.3])
    out, S = ref.decay(q, k, v, g, 1.0)
    a, Sa = ref.decay(q[:, :5], k[:, :5], v[:, :5], g, 1.0)
    b, Sb = ref.decay(q[:, 5:], k[:, 5:], v[:, 5:], g, 1.0, Sa)
    assert torch.allclose(torch.cat([a, b], 1), out, rtol=1e-13, atol=1e-13)
    assert torch.allclose(Sb, S, rtol=1e-13, atol=1e-13)


def _differences(f, x, eps=1e-6):
    out = torch.zeros_like(x)
    flat, o = x.reshape(-1), out.reshape(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + eps
        up = f()
        flat[i] = keep - eps
        o[i] = (up - f()) / (2 * eps)
        flat[i] = keep
    return out


@pytest.mark.parametrize("H,K", [(1, 1), (4, 2)])
def test_decay_gradients_are_differences(H, K):
    n, d = 6, 3
    q, k, v, do = _randn(0, H, n, d), _randn(1, K, n, d), _randn(2, K, n, d), _randn(5, H, n, d)
    g, S0, dS = -_randn(4, K).abs(), _randn(3, K, d, d), _randn(6, K, d, d)

    def loss():
        out, S = ref.decay(q, k, v, g, 0.7, S0)
        return ((out * do).sum() + (S * dS).sum()).item()

    grads = ref.decay_backward(q, k, v, g, do, 0.7, S0, dS)
    for x, got in zip((q, k, v, g, S0), grads):
        assert torch.allclose(got, _differences(loss, x), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rotary", [0, 4, 8])
def test_rope_gradients_are_differences(adjacent, rotary):
    x, w, dy = _randn(0, 2, 3, 8), 1 + 0.1 * _randn(1, 2, 8), _randn(2, 2, 3, 8)
    pos = torch.tensor([0, 5, 1000])
    loss = lambda: (ref.rope(x, w, pos, rotary, adjacent=adjacent) * dy).sum().item()
    dx, dw = ref.rope_backward(x, w, pos, dy, rotary, adjacent=adjacent)
    assert torch.allclose(dx, _differences(loss, x), rtol=1e-6, atol=1e-7)
    assert torch.allclose(dw, _differences(loss, w), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_turns_pairs_by_the_difference_of_positions(adjacent):
    """Products of a query and a key depend on their distance alone."""
    q, k = _randn(0, 1, 1, 8), _randn(1, 1, 1, 8)
    dot = lambda i, j: (ref.rope(q, None, torch.tensor([i]), 8, adjacent=adjacent)
                        * ref.rope(k, None, torch.tensor([j]), 8, adjacent=adjacent)).sum()
    assert torch.allclose(dot(3, 1), dot(103, 101), rtol=1e-12)
    assert not torch.allclose(dot(3, 1), dot(3, 2), rtol=1e-3)
