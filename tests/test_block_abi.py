"""The decoder block's operators: refusals of the C entry points and of the Python binding, and
the workspace sizes.  No kernel runs: every call below fails on the host."""
import ctypes

import pytest
import torch

from paper_2606_07317_amd import gbla

P = 0x10000          # fake, 256-byte aligned device address; never dereferenced
MIS = 0x10008
ODD = 0x10002


@pytest.fixture(scope="module")
def lib():
    return gbla.load_library()


def delta_shape(**kw):
    base = dict(batch=2, seqlen=1000, heads=4, value_heads=8, head_dim=64, max_seqlen=0,
                dtype=gbla.GBLA_BF16, scale=0.125)
    base.update(kw)
    return gbla.DeltaShape(**base)


def norm_shape(**kw):
    base = dict(rows=10, width=1024, dtype=gbla.GBLA_BF16, out_dtype=gbla.GBLA_BF16, group=0, eps=1e-6)
    base.update(kw)
    return gbla.NormShape(**base)


BAD_DELTA = [(dict(batch=0), 1), (dict(seqlen=-1), 1), (dict(heads=0), 1), (dict(value_heads=0), 1),
             (dict(value_heads=6), 1), (dict(value_heads=2), 1), (dict(scale=float("inf")), 1),
             (dict(scale=float("nan")), 1), (dict(head_dim=96), 2), (dict(dtype=gbla.GBLA_E4M3), 2),
             (dict(heads=1, value_heads=65536), 2)]
BAD_NORM = [(dict(rows=-1), 1), (dict(width=0), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
            (dict(eps=float("inf")), 1), (dict(width=12), 2), (dict(width=16392), 2), (dict(dtype=gbla.GBLA_E4M3), 2),
            (dict(dtype=7), 2), (dict(rows=1 << 62), 2)]
BAD_NORM_OUT = [(dict(group=-1), 1), (dict(out_dtype=gbla.GBLA_F32), 2), (dict(group=128), 2),
                (dict(out_dtype=gbla.GBLA_E4M3, group=64), 2), (dict(out_dtype=gbla.GBLA_E4M3, group=128, width=1032), 2)]


def _fill(names, first, given):
    return [given.get(n, d) for n, d in zip(names, first)]


def forward(lib, s, ws_bytes=1 << 40, **p):
    a = _fill("q k v g b S0 cu ws".split(), (P, P, P, P, P, None, None, P), p)
    b = _fill(("out", "S"), (P, None), p)
    return lib.gbla_delta_forward(None if s is None else ctypes.byref(s), *a, ws_bytes, *b, None)


def backward(lib, s, ws_bytes=1 << 40, **p):
    a = _fill("q k v g b S0 cu do dS ws".split(), (P, P, P, P, P, None, None, P, None, P), p)
    b = _fill("dq dk dv dg db dS0".split(), (P, P, P, P, P, None), p)
    return lib.gbla_delta_backward(None if s is None else ctypes.byref(s), *a, ws_bytes, *b, None)


def step(lib, s, slots=2, **p):
    a = _fill("q k v g b idx".split(), (P, P, P, P, P, P), p)
    b = _fill(("state", "out"), (P, P), p)
    return lib.gbla_delta_step(None if s is None else ctypes.byref(s), *a, slots, *b, None)


def norm(lib, s, **p):
    a = _fill("x res w sum out scales".split(), (P, P, P, P, P, P), p)
    return lib.gbla_add_norm(None if s is None else ctypes.byref(s), *a, None)


def norm_back(lib, s, ws_bytes=1 << 40, **p):
    a = _fill("sum w dy ds ws".split(), (P, P, P, P, P), p)
    b = _fill(("dx", "dw"), (P, P), p)
    return lib.gbla_add_norm_backward(None if s is None else ctypes.byref(s), *a, ws_bytes, *b, None)


@pytest.mark.parametrize("change,status", BAD_DELTA)
def test_delta_refuses_shapes(lib, change, status):
    s = delta_shape(**change)
    assert forward(lib, s) == status and backward(lib, s) == status
    assert step(lib, delta_shape(**{"seqlen": 1, **change})) == status
    for f in (lib.gbla_delta_workspace_bytes, lib.gbla_delta_backward_workspace_bytes,
              lib.gbla_delta_ragged_workspace_bytes, lib.gbla_delta_backward_ragged_workspace_bytes):
        assert f(ctypes.byref(s)) == 0


def test_delta_refuses_arrays(lib):
    s = delta_shape()
    assert forward(lib, None) == 1 and backward(lib, None) == 1 and step(lib, None) == 1
    assert forward(lib, delta_shape(max_seqlen=-1), cu=P) == 1
    for name in ("q", "k", "v", "g", "b", "out"):
        assert forward(lib, s, **{name: None}) == 1, name
    for name in ("q", "k", "v", "out", "S0", "S"):
        assert forward(lib, s, **{name: MIS}) == 3, name
    for name in ("g", "b", "cu"):
        assert forward(lib, s, **{name: ODD}) == 3, name
    for name in ("q", "k", "v", "g", "b", "do", "dq", "dk", "dv", "dg", "db"):
        assert backward(lib, s, **{name: None}) == 1, name
    for name in ("q", "k", "v", "do", "dq", "dk", "dv", "S0", "dS", "dS0"):
        assert backward(lib, s, **{name: MIS}) == 3, name
    for name in ("g", "b", "cu", "dg", "db"):
        assert backward(lib, s, **{name: ODD}) == 3, name
    for call, size in ((forward, lib.gbla_delta_workspace_bytes), (backward, lib.gbla_delta_backward_workspace_bytes)):
        assert call(lib, s, ws=None) == 4 and call(lib, s, ws=P + 64) == 3
        assert call(lib, s, ws_bytes=size(ctypes.byref(s)) // 2) == 4


def test_delta_step_refuses(lib):
    s = delta_shape(seqlen=1)
    for name in ("q", "k", "v", "g", "b", "state", "out"):
        assert step(lib, s, **{name: None}) == 1, name
    for name in ("q", "k", "v", "state", "out"):
        assert step(lib, s, **{name: MIS}) == 3, name
    for name in ("g", "b", "idx"):
        assert step(lib, s, **{name: ODD}) == 3, name
    assert step(lib, s, slots=0) == 1
    assert step(lib, s, slots=1, idx=None) == 1      # row 1 has no slot
    assert step(lib, delta_shape(seqlen=2)) == 1


def test_delta_workspace_sizes(lib):
    for f in (lib.gbla_delta_workspace_bytes, lib.gbla_delta_backward_workspace_bytes,
              lib.gbla_delta_ragged_workspace_bytes, lib.gbla_delta_backward_ragged_workspace_bytes):
        sizes = {f(ctypes.byref(delta_shape(max_seqlen=m))) for m in (0, 1, 700, 1000)}
        assert len(sizes) == 1 and sizes.pop() % 256 == 0
        assert f(ctypes.byref(delta_shape(seqlen=0))) > 0
        assert f(None) == 0
    many = ctypes.byref(delta_shape(batch=64, seqlen=177929))
    assert lib.gbla_delta_ragged_workspace_bytes(many) < lib.gbla_delta_workspace_bytes(many) // 8
    need = lib.gbla_delta_ragged_workspace_bytes(many)
    assert forward(lib, delta_shape(batch=64, seqlen=177929), ws_bytes=need - 1, cu=P) == 4
    with pytest.raises(gbla.GblaError):
        gbla.delta_workspace_bytes(delta_shape(batch=0))
    with pytest.raises(gbla.GblaError):
        gbla.delta_backward_workspace_bytes(delta_shape(batch=0), ragged=True)


@pytest.mark.parametrize("change,status", BAD_NORM)
def test_norm_refuses_shapes(lib, change, status):
    s = norm_shape(**{"out_dtype": change.get("dtype", gbla.GBLA_BF16), **change})
    assert norm(lib, s) == status and norm_back(lib, s) == status
    assert lib.gbla_add_norm_backward_workspace_bytes(ctypes.byref(s)) == 0


@pytest.mark.parametrize("change,status", BAD_NORM_OUT)
def test_norm_refuses_outputs(lib, change, status):
    assert norm(lib, norm_shape(**change)) == status


def test_norm_refuses_arrays(lib):
    s = norm_shape()
    assert norm(lib, None) == 1 and norm_back(lib, None) == 1
    for name in ("x", "w", "out"):
        assert norm(lib, s, **{name: None}) == 1, name
    for name in ("x", "res", "w", "sum", "out"):
        assert norm(lib, s, **{name: MIS}) == 3, name
    eight = norm_shape(out_dtype=gbla.GBLA_E4M3, group=128)
    assert norm(lib, eight, scales=None) == 1 and norm(lib, eight, scales=ODD) == 3
    for name in ("sum", "w", "dy", "dx", "dw"):
        assert norm_back(lib, s, **{name: None}) == 1, name
    for name in ("sum", "w", "dy", "ds", "dx", "dw"):
        assert norm_back(lib, s, **{name: MIS}) == 3, name
    assert norm_back(lib, s, ws=None) == 4 and norm_back(lib, s, ws=P + 64) == 3
    assert norm_back(lib, s, ws_bytes=lib.gbla_add_norm_backward_workspace_bytes(ctypes.byref(s)) - 1) == 4
    with pytest.raises(gbla.GblaError):
        gbla.add_rms_norm_backward_workspace_bytes(norm_shape(width=12))


def test_python_refuses_cpu_tensors():
    x, v, g = torch.zeros(1, 2, 3, 32), torch.zeros(1, 4, 3, 32), torch.zeros(1, 4, 3)
    with pytest.raises(ValueError, match="GPU"):
        gbla.delta_attention(x, x, v, g, g)
    with pytest.raises(ValueError, match="GPU"):
        gbla.delta_attention_backward(x, x, v, g, g, v)
    with pytest.raises(ValueError, match="GPU"):
        gbla.delta_step(x[0], x[0], v[0], g[0], g[0], torch.zeros(2, 4, 32, 32))
    for call in (lambda: gbla.add_rms_norm(x, g), lambda: gbla.add_rms_norm_e4m3(x, g),
                 lambda: gbla.add_rms_norm_backward(x, g, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
