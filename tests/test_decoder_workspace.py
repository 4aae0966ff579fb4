"""Scratch sizes of the decoder's operators for packed batches.  Host arithmetic only."""
import ctypes

import pytest

from paper_2606_07317_amd import gbla


@pytest.fixture(scope="module")
def lib():
    return gbla.load_library()


def _decay(N, T, K=16, d=128, max_seqlen=0):
    return gbla.DecayShape(N, T, K, K, d, max_seqlen, gbla.GBLA_BF16, d ** -0.5)


def _rope(N, T, H=16, d=128, flags=0):
    return gbla.RopeShape(N, T, H, H, d, d, gbla.GBLA_BF16, 1e-6, 1e4, flags)


@pytest.mark.parametrize("N,T", [(1, 1), (16, 57511), (64, 177929), (2100, 1075200)])
def test_a_packed_batch_needs_what_its_own_tokens_do(lib, N, T):
    """A record for each unit of at least 128 tokens and each sequence, and no more."""
    for d in (32, 64, 128):
        s = ctypes.byref(_decay(N, T, d=d))
        record = 4 * 16 * d * d
        forward = lib.gbla_decay_ragged_workspace_bytes(s)
        backward = lib.gbla_decay_backward_ragged_workspace_bytes(s)
        assert 0 < forward <= (T // 128 + N) * record + 256
        assert 2 * forward <= backward <= (T // 128 + N) * (2 * record + 2 * 16 * 64) + 3 * 256
        # the two readings cover it
        assert forward <= lib.gbla_decay_workspace_bytes(s)
        assert backward <= lib.gbla_decay_backward_workspace_bytes(s)
        r = ctypes.byref(_rope(N, T, d=d))
        partial = lib.gbla_qk_norm_rope_backward_ragged_workspace_bytes(r)
        # a sum per workgroup of a pass of 256 / (d / 8) tokens
        assert 256 <= partial <= max(256, (T // (2048 // d) + 1) * 32 * d * 4 + 256)
        assert partial <= lib.gbla_qk_norm_rope_backward_workspace_bytes(r)


def test_one_size_whatever_the_bound_of_the_lengths(lib):
    for f in (lib.gbla_decay_ragged_workspace_bytes, lib.gbla_decay_backward_ragged_workspace_bytes):
        assert len({f(ctypes.byref(_decay(64, 177929, max_seqlen=m))) for m in (0, 1, 5000, 177929)}) == 1


def test_refused_shapes_have_no_size(lib):
    for bad in (_decay(0, 10), _decay(1, -1), _decay(1, 10, d=48), _decay(1, 10, max_seqlen=-1)):
        assert lib.gbla_decay_ragged_workspace_bytes(ctypes.byref(bad)) == 0
        assert lib.gbla_decay_backward_ragged_workspace_bytes(ctypes.byref(bad)) == 0
    for bad in (_rope(0, 10), _rope(1, 10, d=48), _rope(1, 10, flags=1)):
        assert lib.gbla_qk_norm_rope_backward_ragged_workspace_bytes(ctypes.byref(bad)) == 0
    assert lib.gbla_decay_ragged_workspace_bytes(None) == 0
    with pytest.raises(gbla.GblaError):
        gbla.decay_workspace_bytes(_decay(0, 10), ragged=True)
    with pytest.raises(gbla.GblaError):
        gbla.decay_backward_workspace_bytes(_decay(0, 10), ragged=True)
    with pytest.raises(gbla.GblaError):
        gbla.qk_norm_rope_backward_workspace_bytes(_rope(0, 10), ragged=True)


def test_the_workspace_that_a_packed_call_asks_for_is_its_own(lib):
    """One byte less is refused, before anything is enqueued."""
    P = 0x10000
    s = _decay(64, 177929)
    need = lib.gbla_decay_ragged_workspace_bytes(ctypes.byref(s))
    call = lambda ws: lib.gbla_decay_forward(ctypes.byref(s), P, P, P, P, None, P, P, ws, P, None, None)
    assert call(need - 1) == 4
    assert gbla.decay_workspace_bytes(s, ragged=True) == need
    assert 50 * need < gbla.decay_workspace_bytes(s)
