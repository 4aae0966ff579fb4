"""The 64-bit references of the decoder block's operators against other forms of the same
mathematics: products of the tokens' maps, central differences, torch's own eight bits."""
import pytest
import torch

from oracle import gbla_block as ref
from oracle import gbla_decoder as dec


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _case(H, V, n, d):
    q, k, v = _randn(0, H, n, d), _randn(1, H, n, d), _randn(2, V, n, d)
    k = k / k.norm(dim=-1, keepdim=True)
    return q, k, v, -_randn(3, V, n).abs(), torch.sigmoid(_randn(4, V, n)), _randn(5, V, d, d)


@pytest.mark.parametrize("H,V", [(1, 1), (2, 4)])
def test_recurrence_is_the_product_of_the_tokens_maps(H, V):
    n, d = 7, 4
    q, k, v, g, b, S0 = _case(H, V, n, d)
    out, S = ref.delta(q, k, v, g, b, 0.5, S0)
    for h in range(V):
        X = S0[h]
        for t in range(n):
            kt = k[h * H // V, t]
            A = torch.exp(g[h, t]) * (torch.eye(d) - b[h, t] * torch.outer(kt, kt))
            X = A @ X + b[h, t] * torch.outer(kt, v[h, t])
            assert torch.allclose(out[h, t], 0.5 * X.T @ q[h * H // V, t], rtol=1e-12, atol=1e-12)
        assert torch.allclose(S[h], X, rtol=1e-12, atol=1e-12)


def test_recurrence_without_correction_is_the_decay_attention():
    """Keys orthogonal to what was written: nothing is read back, so beta k v^T is added."""
    n = d = 6
    q, v = _randn(0, 1, n, d), _randn(2, 1, n, d)
    k = torch.eye(d, dtype=torch.float64)[None]
    g, b = torch.full((1, n), -0.3), torch.ones(1, n)
    a, S = ref.delta(q, k, v, g, b, 0.7)
    c, T = dec.decay(q, k, v, torch.tensor([-0.3]), 0.7)
    assert torch.allclose(a, c, rtol=1e-12, atol=1e-12) and torch.allclose(S, T, rtol=1e-12, atol=1e-12)


def test_a_token_written_with_strength_one_is_read_back():
    q, k, v, g, b, S0 = _case(1, 1, 5, 8)
    b[:] = 1.0
    out, _ = ref.delta(k, k, v, g, b, 1.0, S0)
    assert torch.allclose(out, v, rtol=1e-10, atol=1e-10)


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


@pytest.mark.parametrize("H,V", [(1, 1), (2, 4)])
def test_delta_gradients_are_differences(H, V):
    n, d = 5, 3
    q, k, v, g, b, S0 = _case(H, V, n, d)
    do, dS = _randn(6, V, n, d), _randn(7, V, d, d)

    def loss():
        out, S = ref.delta(q, k, v, g, b, 0.7, S0)
        return ((out * do).sum() + (S * dS).sum()).item()

    for x, got in zip((q, k, v, g, b, S0), ref.delta_backward(q, k, v, g, b, do, 0.7, S0, dS)):
        assert torch.allclose(got, _differences(loss, x), rtol=1e-6, atol=1e-7)


def test_sizes_bound_a_perturbed_run():
    """Values off by a relative 1e-3 move results by no more than 1e-3 of the sizes."""
    q, k, v, g, b, S0 = _case(2, 4, 150, 8)
    out, S = ref.delta(q, k, v, g, b, 0.5, S0)
    off = v * (1 + 1e-3 * torch.sign(_randn(9, *v.shape)))
    a, T = ref.delta(q, k, off, g, b, 0.5, S0)
    so, sS = ref.delta_sizes(q, k, v, g, b, 0.5, S0)
    assert ((a - out).abs() <= 1e-3 * so).all() and ((T - S).norm(dim=1, keepdim=True) <= 1e-3 * sS).all()


@pytest.mark.parametrize("with_ds", [False, True])
def test_norm_gradients_are_differences(with_ds):
    s, w, dy = _randn(0, 3, 8), 1 + 0.1 * _randn(1, 8), _randn(2, 3, 8)
    ds = _randn(3, 3, 8) if with_ds else None

    def loss():
        y, t = ref.add_norm(s, None, w, 1e-3)
        return ((y * dy).sum() + (0.0 if ds is None else (t * ds).sum())).item()

    for x, got in zip((s, w), ref.add_norm_backward(s, w, dy, ds, 1e-3)):
        assert torch.allclose(got, _differences(loss, x), rtol=1e-6, atol=1e-7)


def test_eight_bits_are_torchs():
    x = torch.cat([_randn(0, 4000) * 100, _randn(1, 4000) * 2.0 ** -8, torch.tensor([0.0, 448.0, -448.0, 2.0 ** -10])])
    x = x.clamp(-448, 448).float()
    assert torch.equal(ref.to_e4m3(x).float(), x.to(torch.float8_e4m3fn).float())
