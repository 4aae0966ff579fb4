"""Python binding of libgbla.so (argument marshalling only).

Every step of the GBLA forward pass runs in the HIP kernels behind the C ABI
declared in ``include/gbla.h``; this module checks tensor metadata, passes
device pointers and the current HIP stream, and turns status codes into
exceptions.  PyTorch provides device memory and streams, nothing else.  If
the library is not built this module raises; there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgbla.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "gbla.h")

GBLA_F32 = 0
GBLA_BF16 = 1
GBLA_E4M3 = 2  # outputs of add_rms_norm_e4m3
# Ablation switches (shape.flags); all three together is plain BLA, Eq. (1).
NO_GATE = 1   # uniform key gates; gate_logits may be None
NO_CONV = 2   # identity Conv1D; conv_w may be None
NO_NORM = 4   # out = o; out_gate and norm_w may be None
BLA = NO_GATE | NO_CONV | NO_NORM
ROPE_PAIRS = 8  # qk_norm_rope: adjacent channels rotate together
STATUS_NAMES = {0: "GBLA_OK", 1: "GBLA_ERR_INVALID_ARGUMENT", 2: "GBLA_ERR_UNSUPPORTED",
                3: "GBLA_ERR_MISALIGNED", 4: "GBLA_ERR_WORKSPACE", 5: "GBLA_ERR_HIP"}


class GblaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s" % (where, STATUS_NAMES.get(status, status)))


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seqlen", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("conv_width", ctypes.c_int32),
                ("max_seqlen", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class LayerShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("conv_width", ctypes.c_int32), ("max_seqlen", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class RopeShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("theta", ctypes.c_float), ("flags", ctypes.c_uint32)]


class DecayShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_seqlen", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class DeltaShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("value_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_seqlen", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class NormShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("group", ctypes.c_int32), ("eps", ctypes.c_float)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libgbla.so and declare its signatures.  Raises if it is missing."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise GblaError(-1, "loading %s (not built: run __graft_entry__.build())" % path)
    lib = ctypes.CDLL(path)
    P = ctypes.c_void_p
    SP = ctypes.POINTER(Shape)
    sz = ctypes.c_size_t
    lib.gbla_workspace_bytes.argtypes = [SP]
    lib.gbla_workspace_bytes.restype = sz
    lib.gbla_forward.argtypes = [SP, P, P, P, P, P, P, P, P, P, sz, P, P]
    lib.gbla_forward.restype = ctypes.c_int
    lib.gbla_forward_timed.argtypes = [SP, P, P, P, P, P, P, P, P, P, sz, P, P, P, P]
    lib.gbla_forward_timed.restype = ctypes.c_int
    lib.gbla_conv1d.argtypes = [SP, P, P, P, P, P, P, P, P, P]
    lib.gbla_conv1d.restype = ctypes.c_int
    lib.gbla_state.argtypes = [SP, P, P, P, P, P, P, sz, P, P, P]
    lib.gbla_state.restype = ctypes.c_int
    lib.gbla_readout.argtypes = [SP, P, P, P, P, P, P, sz, P, P]
    lib.gbla_readout.restype = ctypes.c_int
    lib.gbla_readout_timed.argtypes = [SP, P, P, P, P, P, P, sz, P, P, P, P]
    lib.gbla_readout_timed.restype = ctypes.c_int
    lib.gbla_forward_noalloc.argtypes = [SP, P, P, P, P, P, P, P, P, P, P]
    lib.gbla_forward_noalloc.restype = ctypes.c_int
    lib.gbla_stream_ceiling.argtypes = [P, P, P, P, P, ctypes.c_int64, ctypes.c_int32, P, P]
    lib.gbla_stream_ceiling.restype = ctypes.c_int
    lib.gbla_backward_workspace_bytes.argtypes = [SP]
    lib.gbla_backward_workspace_bytes.restype = sz
    lib.gbla_backward.argtypes = [SP, P, P, P, P, P, P, P, P, P, P, sz, P, P, P, P, P, P, P, P]
    lib.gbla_backward.restype = ctypes.c_int
    LP = ctypes.POINTER(LayerShape)
    lib.gbla_layer_workspace_bytes.argtypes = [LP]
    lib.gbla_layer_workspace_bytes.restype = sz
    lib.gbla_layer_project.argtypes = [LP, P, P, P, P, P, sz, P, P, P, P, P, P]
    lib.gbla_layer_project.restype = ctypes.c_int
    lib.gbla_layer_forward.argtypes = [LP, P, P, P, P, P, P, sz, P, P]
    lib.gbla_layer_forward.restype = ctypes.c_int
    RP, DP = ctypes.POINTER(RopeShape), ctypes.POINTER(DecayShape)
    lib.gbla_qk_norm_rope.argtypes = [RP] + [P] * 9
    lib.gbla_qk_norm_rope.restype = ctypes.c_int
    for name in ("gbla_qk_norm_rope_backward_workspace_bytes",
                 "gbla_qk_norm_rope_backward_ragged_workspace_bytes"):
        getattr(lib, name).argtypes = [RP]
        getattr(lib, name).restype = sz
    lib.gbla_qk_norm_rope_backward.argtypes = [RP] + [P] * 9 + [sz] + [P] * 5
    lib.gbla_qk_norm_rope_backward.restype = ctypes.c_int
    for name in ("gbla_decay_workspace_bytes", "gbla_decay_backward_workspace_bytes",
                 "gbla_decay_ragged_workspace_bytes", "gbla_decay_backward_ragged_workspace_bytes"):
        getattr(lib, name).argtypes = [DP]
        getattr(lib, name).restype = sz
    lib.gbla_decay_forward.argtypes = [DP] + [P] * 7 + [sz] + [P] * 3
    lib.gbla_decay_forward.restype = ctypes.c_int
    lib.gbla_decay_backward.argtypes = [DP] + [P] * 9 + [sz] + [P] * 6
    lib.gbla_decay_backward.restype = ctypes.c_int
    lib.gbla_decay_step.argtypes = [DP] + [P] * 5 + [ctypes.c_int32] + [P] * 3
    lib.gbla_decay_step.restype = ctypes.c_int
    EP = ctypes.POINTER(DeltaShape)
    for name in ("gbla_delta_workspace_bytes", "gbla_delta_backward_workspace_bytes",
                 "gbla_delta_ragged_workspace_bytes", "gbla_delta_backward_ragged_workspace_bytes"):
        getattr(lib, name).argtypes = [EP]
        getattr(lib, name).restype = sz
    lib.gbla_delta_forward.argtypes = [EP] + [P] * 8 + [sz] + [P] * 3
    lib.gbla_delta_forward.restype = ctypes.c_int
    lib.gbla_delta_backward.argtypes = [EP] + [P] * 10 + [sz] + [P] * 7
    lib.gbla_delta_backward.restype = ctypes.c_int
    lib.gbla_delta_step.argtypes = [EP] + [P] * 6 + [ctypes.c_int32] + [P] * 3
    lib.gbla_delta_step.restype = ctypes.c_int
    NP = ctypes.POINTER(NormShape)
    lib.gbla_add_norm.argtypes = [NP] + [P] * 7
    lib.gbla_add_norm.restype = ctypes.c_int
    lib.gbla_add_norm_backward_workspace_bytes.argtypes = [NP]
    lib.gbla_add_norm_backward_workspace_bytes.restype = sz
    lib.gbla_add_norm_backward.argtypes = [NP] + [P] * 5 + [sz] + [P] * 3
    lib.gbla_add_norm_backward.restype = ctypes.c_int
    lib.gbla_status_string.argtypes = [ctypes.c_int]
    lib.gbla_status_string.restype = ctypes.c_char_p
    if path == LIB_PATH:
        _lib = lib
    return lib


def declared_functions(header: str = HEADER_PATH):
    """Names of the functions that include/gbla.h declares."""
    text = open(header).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(gbla_[a-z0-9_]+)\s*\(", text)))


# ---------------------------------------------------------------------------
# Tensor marshalling.
# ---------------------------------------------------------------------------
def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return GBLA_BF16
    if t.dtype == torch.float32:
        return GBLA_F32
    raise TypeError("activations must be bfloat16 or float32, got %s" % t.dtype)


def _check(t: torch.Tensor, name: str, dtype=None, device=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))


def _check_out(out: torch.Tensor, shape, dev, name: str = "out"):
    """An output buffer the kernels write in full: fp32, contiguous, on the
    device of the inputs, with exactly the expected shape."""
    _check(out, name, torch.float32, dev)
    if tuple(out.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(out.shape), tuple(shape)))


def _check_ws(ws: torch.Tensor, dev, need: int, name: str = "workspace"):
    """Caller-supplied scratch: a contiguous uint8 tensor on the inputs'
    device, at least ``need`` bytes (the library checks the size and the
    256-byte alignment again)."""
    _check(ws, name, torch.uint8, dev)
    if ws.numel() < need:
        raise ValueError("%s holds %d bytes, %d needed" % (name, ws.numel(), need))


def make_shape(q: torch.Tensor, conv_w: Optional[torch.Tensor], eps: float,
               cu_seqlens: Optional[torch.Tensor], max_seqlen: Optional[int],
               flags: int = 0) -> Shape:
    if cu_seqlens is None:
        if q.dim() != 4:
            raise ValueError("dense q must be [B, H, n, d]")
        B, H, n, d = q.shape
        batch, rows, msl = B, n, 0
    else:
        if q.dim() != 3:
            raise ValueError("ragged q must be [H, T, d]")
        H, rows, d = q.shape
        batch = cu_seqlens.numel() - 1
        msl = int(max_seqlen) if max_seqlen is not None else rows
    if conv_w is None:
        if not flags & NO_CONV:
            raise ValueError("conv_w is required unless flags has NO_CONV")
        W = 1  # identity conv
    else:
        if conv_w.dim() != 4 or tuple(conv_w.shape[:3]) != (3, H, d):
            raise ValueError("conv_w must be [3, H, d, W]")
        W = conv_w.shape[3]
    return Shape(batch, H, rows, d, W, msl, _dtype_code(q), float(eps), int(flags))


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _raise(st: int, where: str):
    if st != 0:
        raise GblaError(st, where)


def workspace_bytes(shape: Shape) -> int:
    n = load_library().gbla_workspace_bytes(ctypes.byref(shape))
    if n == 0:
        raise GblaError(1, "gbla_workspace_bytes")
    return int(n)


def alloc_workspace(shape: Shape, device) -> torch.Tensor:
    """Caller-owned scratch for gbla_forward / gbla_state (256-byte aligned)."""
    return torch.empty(workspace_bytes(shape), dtype=torch.uint8, device=device)


def _check_inputs(q, k, v, a, r, conv_w, norm_w, cu_seqlens):
    dev = q.device
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (r, "out_gate")):
        if t is not None:
            _check(t, nm, q.dtype, dev)
            if t.shape != q.shape:
                raise ValueError("%s has shape %s, expected %s" % (nm, tuple(t.shape), tuple(q.shape)))
    if a is not None:
        _check(a, "gate_logits", q.dtype, dev)
        if a.shape != q.shape[:-1]:
            raise ValueError("gate_logits must have shape %s" % (tuple(q.shape[:-1]),))
    if conv_w is not None:
        _check(conv_w, "conv_w", torch.float32, dev)
    if norm_w is not None:
        _check(norm_w, "norm_w", torch.float32, dev)
        if norm_w.shape != (q.shape[-3], q.shape[-1]):
            raise ValueError("norm_w must be [H, d]")
    if cu_seqlens is not None:
        _check(cu_seqlens, "cu_seqlens", torch.int32, dev)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def forward(q, k, v, gate_logits, out_gate, conv_w, norm_w, eps: float = 1e-6,
            cu_seqlens=None, max_seqlen=None, workspace=None, out=None, stream=None,
            flags: int = 0, kernel_events=None) -> torch.Tensor:
    """y = GBLA(q, k, v, a, r) on the GPU (o under NO_NORM); see include/gbla.h
    for the layouts and the ablation switches in ``flags``.
    ``max_seqlen`` (ragged) is an upper bound of the lengths; the default is T.
    It only chooses kernels, and decides a factor of two or more for batches of
    short sequences (d = 32 and 64): with a tight bound they take one launch, whose
    sums round in another order than the three launches of a loose one.
    ``kernel_events`` = (start, stop) torch.cuda.Events recorded just before
    the pass's first kernel and as its last kernel ends (gbla_forward_timed);
    each must have been recorded once before, so that its HIP event exists."""
    _check_inputs(q, k, v, gate_logits, out_gate, conv_w, norm_w, cu_seqlens)
    shape = make_shape(q, conv_w, eps, cu_seqlens, max_seqlen, flags)
    if workspace is None:
        workspace = alloc_workspace(shape, q.device)
    _check_ws(workspace, q.device, workspace_bytes(shape))
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check_out(out, q.shape, q.device)
    args = (ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits), _ptr(out_gate),
            _ptr(conv_w), _ptr(norm_w), _ptr(cu_seqlens), _ptr(workspace), workspace.numel(),
            _ptr(out), _stream(stream))
    if kernel_events is None:
        _raise(load_library().gbla_forward(*args), "gbla_forward")
    else:
        handles = [e.cuda_event for e in kernel_events]
        if not all(handles):
            raise ValueError("kernel_events must have been recorded once before")
        _raise(load_library().gbla_forward_timed(*args, *handles), "gbla_forward_timed")
    return out


NOALLOC_SCRATCH_BYTES = 16 << 20  # GBLA_NOALLOC_SCRATCH_BYTES


def forward_noalloc(q, k, v, gate_logits, out_gate, conv_w, norm_w, eps: float = 1e-6,
                    cu_seqlens=None, max_seqlen=None, out=None, stream=None,
                    flags: int = 0) -> torch.Tensor:
    """gbla_forward_noalloc: the forward with the library's fixed device
    scratch instead of a workspace (for callers that cannot allocate; give
    ``out`` to allocate nothing here either)."""
    _check_inputs(q, k, v, gate_logits, out_gate, conv_w, norm_w, cu_seqlens)
    shape = make_shape(q, conv_w, eps, cu_seqlens, max_seqlen, flags)
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check_out(out, q.shape, q.device)
    st = load_library().gbla_forward_noalloc(
        ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits), _ptr(out_gate),
        _ptr(conv_w), _ptr(norm_w), _ptr(cu_seqlens), _ptr(out), _stream(stream))
    _raise(st, "gbla_forward_noalloc")
    return out


def conv1d(q, k, v, conv_w, cu_seqlens=None, max_seqlen=None, stream=None, flags: int = 0
           ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The Conv1D alone: fp32 q_t, k_t, v_t in the layout of q."""
    _check_inputs(q, k, v, None, None, conv_w, None, cu_seqlens)
    shape = make_shape(q, conv_w, 0.0, cu_seqlens, max_seqlen, flags)
    outs = [torch.empty(q.shape, dtype=torch.float32, device=q.device) for _ in range(3)]
    st = load_library().gbla_conv1d(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                                    _ptr(cu_seqlens), *[_ptr(o) for o in outs], _stream(stream))
    _raise(st, "gbla_conv1d")
    return tuple(outs)


def state(k, v, gate_logits, conv_w, cu_seqlens=None, max_seqlen=None, workspace=None,
          stream=None, flags: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
    """The normalised global state S [N,H,d,d] and z [N,H,d] (fp32)."""
    _check_inputs(k, k, v, gate_logits, None, conv_w, None, cu_seqlens)
    shape = make_shape(k, conv_w, 0.0, cu_seqlens, max_seqlen, flags)
    if workspace is None:
        workspace = alloc_workspace(shape, k.device)
    _check_ws(workspace, k.device, workspace_bytes(shape))
    N, H, d = shape.batch, shape.heads, shape.head_dim
    S = torch.empty((N, H, d, d), dtype=torch.float32, device=k.device)
    z = torch.empty((N, H, d), dtype=torch.float32, device=k.device)
    st = load_library().gbla_state(ctypes.byref(shape), _ptr(k), _ptr(v), _ptr(gate_logits),
                                   _ptr(conv_w), _ptr(cu_seqlens), _ptr(workspace),
                                   workspace.numel(), _ptr(S), _ptr(z), _stream(stream))
    _raise(st, "gbla_state")
    return S, z


def readout(q, out_gate, conv_w, norm_w, workspace, eps: float = 1e-6, cu_seqlens=None,
            max_seqlen=None, out=None, stream=None, flags: int = 0,
            kernel_events=None) -> torch.Tensor:
    """Readout + gated RMSNorm from the state a preceding state() call left in
    ``workspace``.  ``kernel_events`` = (start, stop) torch.cuda.Events that
    are recorded when the readout kernel begins and ends (gbla_readout_timed);
    each must have been recorded once before, so that its HIP event exists."""
    _check_inputs(q, None, None, None, out_gate, conv_w, norm_w, cu_seqlens)
    shape = make_shape(q, conv_w, eps, cu_seqlens, max_seqlen, flags)
    _check_ws(workspace, q.device, workspace_bytes(shape))
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check_out(out, q.shape, q.device)
    args = (ctypes.byref(shape), _ptr(q), _ptr(out_gate), _ptr(conv_w), _ptr(norm_w),
            _ptr(cu_seqlens), _ptr(workspace), workspace.numel(), _ptr(out), _stream(stream))
    if kernel_events is None:
        _raise(load_library().gbla_readout(*args), "gbla_readout")
    else:
        handles = [e.cuda_event for e in kernel_events]
        if not all(handles):
            raise ValueError("kernel_events must have been recorded once before")
        _raise(load_library().gbla_readout_timed(*args, *handles), "gbla_readout_timed")
    return out


def stream_ceiling(q, k, v, gate_logits, out_gate, out=None, stream=None) -> torch.Tensor:
    """Measurement aid (gbla_stream_ceiling): one launch that moves the
    forward's bytes for these bf16 tensors (q, k, v, out_gate read, one logit
    per token read, fp32 out written) with none of its arithmetic."""
    dev = q.device
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out_gate, "out_gate")):
        _check(t, nm, torch.bfloat16, dev)
        if t.shape != q.shape:
            raise ValueError("%s must have the shape of q" % nm)
    _check(gate_logits, "gate_logits", torch.bfloat16, dev)
    if gate_logits.shape != q.shape[:-1]:
        raise ValueError("gate_logits must have shape %s" % (tuple(q.shape[:-1]),))
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=dev)
    _check_out(out, q.shape, dev)
    d = q.shape[-1]
    st = load_library().gbla_stream_ceiling(_ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits),
                                            _ptr(out_gate), q.numel() // d, d, _ptr(out),
                                            _stream(stream))
    _raise(st, "gbla_stream_ceiling")
    return out


def backward_workspace_bytes(shape: Shape) -> int:
    n = load_library().gbla_backward_workspace_bytes(ctypes.byref(shape))
    if n == 0:
        raise GblaError(1, "gbla_backward_workspace_bytes")
    return int(n)


def backward(q, k, v, gate_logits, out_gate, conv_w, norm_w, dy, eps: float = 1e-6,
             cu_seqlens=None, max_seqlen=None, workspace=None, stream=None,
             grads: Optional[dict] = None, flags: int = 0) -> dict:
    """Gradients of sum(forward(...) * dy) with respect to every input (fp32):
    a dict with dq, dk, dv, da (gate logits), dr (out gate), dconv_w, dgamma
    (norm weight), shaped like the inputs.  ``grads`` may hold preallocated
    fp32 outputs under those names; they are overwritten.  Under the ablation
    switches in ``flags`` the removed inputs may be None and their gradients
    are left out of the dict."""
    _check_inputs(q, k, v, gate_logits, out_gate, conv_w, norm_w, cu_seqlens)
    dev = q.device
    _check(dy, "dy", torch.float32, dev)
    if dy.shape != q.shape:
        raise ValueError("dy must have the shape of q")
    shape = make_shape(q, conv_w, eps, cu_seqlens, max_seqlen, flags)
    if workspace is None:
        workspace = torch.empty(backward_workspace_bytes(shape), dtype=torch.uint8, device=dev)
    _check_ws(workspace, dev, backward_workspace_bytes(shape))
    f32 = dict(dtype=torch.float32, device=dev)
    want = {n: q.shape for n in ("dq", "dk", "dv")}
    if not flags & NO_NORM:
        want.update(dr=q.shape, dgamma=norm_w.shape)
    if not flags & NO_GATE:
        want.update(da=q.shape[:-1])
    if not flags & NO_CONV:
        want.update(dconv_w=conv_w.shape)
    g = dict(grads or {})
    for n, shp in want.items():
        if n not in g:
            g[n] = torch.empty(shp, **f32)
        _check(g[n], n, torch.float32, dev)
        if g[n].shape != shp:
            raise ValueError("%s must have shape %s" % (n, tuple(shp)))
    st = load_library().gbla_backward(
        ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits), _ptr(out_gate),
        _ptr(conv_w), _ptr(norm_w), _ptr(cu_seqlens), _ptr(dy), _ptr(workspace), workspace.numel(),
        _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]), _ptr(g.get("da")), _ptr(g.get("dr")),
        _ptr(g.get("dconv_w")), _ptr(g.get("dgamma")), _stream(stream))
    _raise(st, "gbla_backward")
    return g


# ---------------------------------------------------------------------------
# The full layer from the embeddings X.
# ---------------------------------------------------------------------------
def layer_shape(x, conv_x, heads: int, head_dim: int, eps: float, cu_seqlens=None,
                max_seqlen=None) -> LayerShape:
    if cu_seqlens is None:
        if x.dim() != 3:
            raise ValueError("dense x must be [B, L, d_model]")
        B, L, dm = x.shape
        batch, rows, msl = B, L, 0
    else:
        if x.dim() != 2:
            raise ValueError("ragged x must be [T, d_model]")
        rows, dm = x.shape
        batch = cu_seqlens.numel() - 1
        msl = int(max_seqlen) if max_seqlen is not None else rows
    if conv_x.dim() != 2 or conv_x.shape[0] != dm:
        raise ValueError("conv_x must be [d_model, W]")
    return LayerShape(batch, rows, dm, heads, head_dim, conv_x.shape[1], msl, _dtype_code(x),
                      float(eps))


def _check_layer(x, conv_x, w_proj, heads, head_dim, cu_seqlens):
    dev = x.device
    _check(x, "x", torch.bfloat16, dev)
    _check(conv_x, "conv_x", torch.float32, dev)
    _check(w_proj, "w_proj", torch.bfloat16, dev)
    if w_proj.shape != (heads * (4 * head_dim + 1), x.shape[-1]):
        raise ValueError("w_proj must be [H*(4*d+1), d_model]")
    if cu_seqlens is not None:
        _check(cu_seqlens, "cu_seqlens", torch.int32, dev)


def layer_project(x, conv_x, w_proj, heads: int, head_dim: int, cu_seqlens=None,
                  max_seqlen=None, workspace=None, stream=None) -> dict:
    """Conv1D on x and the stacked projections: bf16 q, k, v, r in the
    attention layout ([B,H,L,d] or [H,T,d]) and the gate logits a."""
    _check_layer(x, conv_x, w_proj, heads, head_dim, cu_seqlens)
    shape = layer_shape(x, conv_x, heads, head_dim, 0.0, cu_seqlens, max_seqlen)
    if workspace is None:
        workspace = torch.empty(layer_workspace_bytes(shape), dtype=torch.uint8, device=x.device)
    _check_ws(workspace, x.device, layer_workspace_bytes(shape))
    if cu_seqlens is None:
        act = (shape.batch, heads, shape.seqlen, head_dim)
    else:
        act = (heads, shape.seqlen, head_dim)
    out = {n: torch.empty(act, dtype=torch.bfloat16, device=x.device) for n in ("q", "k", "v", "r")}
    out["a"] = torch.empty(act[:-1], dtype=torch.bfloat16, device=x.device)
    st = load_library().gbla_layer_project(
        ctypes.byref(shape), _ptr(x), _ptr(conv_x), _ptr(w_proj), _ptr(cu_seqlens), _ptr(workspace),
        workspace.numel(), _ptr(out["q"]), _ptr(out["k"]), _ptr(out["v"]), _ptr(out["r"]),
        _ptr(out["a"]), _stream(stream))
    _raise(st, "gbla_layer_project")
    return out


def layer_workspace_bytes(shape: LayerShape) -> int:
    n = load_library().gbla_layer_workspace_bytes(ctypes.byref(shape))
    if n == 0:
        raise GblaError(1, "gbla_layer_workspace_bytes")
    return int(n)


def layer_forward(x, conv_x, w_proj, norm_w, eps: float = 1e-6, cu_seqlens=None,
                  max_seqlen=None, workspace=None, out=None, stream=None) -> torch.Tensor:
    """The whole layer from the embeddings x; y in the attention layout."""
    if norm_w.dim() != 2:
        raise ValueError("norm_w must be [H, d]")
    heads, head_dim = norm_w.shape
    _check_layer(x, conv_x, w_proj, heads, head_dim, cu_seqlens)
    _check(norm_w, "norm_w", torch.float32, x.device)
    shape = layer_shape(x, conv_x, heads, head_dim, eps, cu_seqlens, max_seqlen)
    if workspace is None:
        workspace = torch.empty(layer_workspace_bytes(shape), dtype=torch.uint8, device=x.device)
    _check_ws(workspace, x.device, layer_workspace_bytes(shape))
    act = ((shape.batch, heads, shape.seqlen, head_dim) if cu_seqlens is None
           else (heads, shape.seqlen, head_dim))
    if out is None:
        out = torch.empty(act, dtype=torch.float32, device=x.device)
    _check_out(out, act, x.device)
    st = load_library().gbla_layer_forward(
        ctypes.byref(shape), _ptr(x), _ptr(conv_x), _ptr(w_proj), _ptr(norm_w), _ptr(cu_seqlens),
        _ptr(workspace), workspace.numel(), _ptr(out), _stream(stream))
    _raise(st, "gbla_layer_forward")
    return out


# ---------------------------------------------------------------------------
# The decoder's operators: norm and rotation of queries and keys, and causal
# linear attention with a decay.
# ---------------------------------------------------------------------------
_HERE = contextlib.nullcontext()


def _on(device, stream):
    """A context in which ``device`` is current and ``stream`` (a torch stream, a HIP
    handle, or None for the device's current one) is its current stream, so that
    what a call allocates belongs to the stream that it runs on."""
    if stream is None:
        return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if not hasattr(stream, "cuda_stream"):
        handle = int(stream)
        stream = (torch.cuda.ExternalStream(handle, device=device) if handle
                  else torch.cuda.default_stream(device))
    if stream.device != device:
        raise ValueError("stream is on %s, the tensors on %s" % (stream.device, device))
    return torch.cuda.stream(stream)


# The handle of a device's current stream: torch's own shortcut where it has one, since
# building a Stream object takes longer (1.9 us) than a small kernel's whole call should.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _current(device) -> int:
    if _raw_stream is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _want(t, name, shape, dtype, device):
    """Refuses a tensor that is not what the call takes; shape: a torch.Size or a tuple.
    ``device`` is one that has been checked already."""
    if (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.device == device
            and t.is_contiguous()):
        return
    _check(t, name, dtype, device)
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))


def _like(t, name, x):
    """``t`` if it can take an output of the shape and type of x, else a new tensor."""
    if t is None:
        return torch.empty_like(x)
    _want(t, name, x.shape, x.dtype, x.device)
    return t


def _size_of(t, dim, at) -> int:
    return t.shape[at] if isinstance(t, torch.Tensor) and t.dim() == dim else 0


def _query_key(q, k, cu_seqlens):
    """Batch, tokens per head, head counts and head dim of q and k, which may have
    different head counts."""
    _check(q, "q")
    dev = q.device
    if cu_seqlens is None:
        if q.dim() != 4:
            raise ValueError("dense q and k must be [B, H, n, d]")
        B, H, n, d = q.shape
        K = _size_of(k, 4, 1)
        _want(k, "k", (B, K, n, d), q.dtype, dev)
        return B, n, H, K, d
    _check(cu_seqlens, "cu_seqlens", torch.int32, dev)
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        raise ValueError("cu_seqlens must be [N + 1]")
    if q.dim() != 3:
        raise ValueError("ragged q and k must be [H, T, d]")
    H, T, d = q.shape
    K = _size_of(k, 3, 0)
    _want(k, "k", (K, T, d), q.dtype, dev)
    return cu_seqlens.numel() - 1, T, H, K, d


def rope_shape(q, k, cu_seqlens=None, rotary_dim=None, theta: float = 10000.0, eps: float = 1e-6,
               flags: int = 0) -> RopeShape:
    B, n, H, K, d = _query_key(q, k, cu_seqlens)
    return RopeShape(B, n, H, K, d, d if rotary_dim is None else int(rotary_dim), _dtype_code(q),
                     float(eps), float(theta), int(flags))


def _check_rope(q, k, q_w, k_w, positions, cu_seqlens, shape):
    dev = q.device
    if not shape.flags & NO_NORM:
        _want(q_w, "q_w", (shape.heads, shape.head_dim), torch.float32, dev)
        _want(k_w, "k_w", (shape.kv_heads, shape.head_dim), torch.float32, dev)
    if positions is not None:
        rows = (shape.batch, shape.seqlen) if cu_seqlens is None else (shape.seqlen,)
        _want(positions, "positions", rows, torch.int32, dev)


def qk_norm_rope(q, k, q_w, k_w, positions=None, cu_seqlens=None, rotary_dim=None,
                 theta: float = 10000.0, eps: float = 1e-6, flags: int = 0, q_out=None, k_out=None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """RMS norm of every head's queries and keys (weights q_w [H, d], k_w [K, d]), then
    the rotation of their first ``rotary_dim`` channels (default: all) by position;
    see include/gbla.h.  q [B, H, n, d] or [H, T, d], k with its own head count;
    ``positions`` int32 [B, n] or [T], by default each token's index in its sequence.
    ``flags``: NO_NORM (q_w, k_w may be None), ROPE_PAIRS.  Returns the rotated q and
    k in their type; ``q_out`` / ``k_out`` may be q / k themselves."""
    shape = rope_shape(q, k, cu_seqlens, rotary_dim, theta, eps, flags)
    _check_rope(q, k, q_w, k_w, positions, cu_seqlens, shape)
    dev = q.device
    with _on(dev, stream):
        q_out = _like(q_out, "q_out", q)
        k_out = _like(k_out, "k_out", k)
        st = load_library().gbla_qk_norm_rope(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(q_w), _ptr(k_w), _ptr(positions),
            _ptr(cu_seqlens), _ptr(q_out), _ptr(k_out), _current(dev))
    _raise(st, "gbla_qk_norm_rope")
    return q_out, k_out


def _scratch(name: str, shape, ragged: bool) -> int:
    name += "_ragged_workspace_bytes" if ragged else "_workspace_bytes"
    n = getattr(load_library(), name)(ctypes.byref(shape))
    if n == 0:
        raise GblaError(1, name)
    return int(n)


def qk_norm_rope_backward_workspace_bytes(shape: RopeShape, ragged: bool = False) -> int:
    """``ragged``: for calls with cu_seqlens only, which take (much) less than both readings."""
    return _scratch("gbla_qk_norm_rope_backward", shape, ragged)


def qk_norm_rope_backward(q, k, q_w, k_w, dq_out, dk_out, positions=None, cu_seqlens=None,
                          rotary_dim=None, theta: float = 10000.0, eps: float = 1e-6,
                          flags: int = 0, workspace=None, grads: Optional[dict] = None,
                          stream=None) -> dict:
    """Gradients of sum(q_out * dq_out) + sum(k_out * dk_out) for the inputs of
    qk_norm_rope: a dict with dq, dk (in q's type) and, unless NO_NORM, dq_w, dk_w
    (fp32).  ``grads`` may hold outputs under those names; dq / dk may be dq_out /
    dk_out themselves."""
    shape = rope_shape(q, k, cu_seqlens, rotary_dim, theta, eps, flags)
    _check_rope(q, k, q_w, k_w, positions, cu_seqlens, shape)
    dev = q.device
    _want(dq_out, "dq_out", q.shape, q.dtype, dev)
    _want(dk_out, "dk_out", k.shape, q.dtype, dev)
    need = qk_norm_rope_backward_workspace_bytes(shape, cu_seqlens is not None)
    g = dict(grads or {})
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        g["dq"] = _like(g.get("dq"), "dq", q)
        g["dk"] = _like(g.get("dk"), "dk", k)
        if not flags & NO_NORM:
            g["dq_w"] = _like(g.get("dq_w"), "dq_w", q_w)
            g["dk_w"] = _like(g.get("dk_w"), "dk_w", k_w)
        st = load_library().gbla_qk_norm_rope_backward(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(q_w), _ptr(k_w), _ptr(positions),
            _ptr(cu_seqlens), _ptr(dq_out), _ptr(dk_out), _ptr(workspace), workspace.numel(),
            _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g.get("dq_w")), _ptr(g.get("dk_w")),
            _current(dev))
    _raise(st, "gbla_qk_norm_rope_backward")
    return g


def decay_shape(q, k, scale: Optional[float] = None, cu_seqlens=None, max_seqlen=None) -> DecayShape:
    B, n, H, K, d = _query_key(q, k, cu_seqlens)
    msl = 0
    if cu_seqlens is not None:
        msl = int(max_seqlen) if max_seqlen is not None else n
    return DecayShape(B, n, H, K, d, msl, _dtype_code(q),
                      float(d) ** -0.5 if scale is None else float(scale))


def decay_workspace_bytes(shape: DecayShape, ragged: bool = False) -> int:
    """``ragged``: for calls with cu_seqlens only, which take (much) less than both readings."""
    return _scratch("gbla_decay", shape, ragged)


def decay_backward_workspace_bytes(shape: DecayShape, ragged: bool = False) -> int:
    return _scratch("gbla_decay_backward", shape, ragged)


def _check_decay(q, k, v, log_decay, shape, states):
    dev = q.device
    _want(v, "v", k.shape, q.dtype, dev)
    _want(log_decay, "log_decay", (shape.kv_heads,), torch.float32, dev)
    for t, name in states:
        if t is not None:
            _want(t, name, (shape.batch, shape.kv_heads, shape.head_dim, shape.head_dim),
                  torch.float32, dev)


def decay_attention(q, k, v, log_decay, scale: Optional[float] = None, initial_state=None,
                    final_state=None, cu_seqlens=None, max_seqlen=None, workspace=None, out=None,
                    stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Causal linear attention with a decay per key head, S_t = exp(g) S_{t-1} +
    k_t v_t^T, o_t = scale S_t^T q_t (scale d^-1/2 by default); see include/gbla.h.
    q [B, H, n, d] or [H, T, d]; k, v with K heads, K dividing H; log_decay [K] fp32,
    <= 0; ``initial_state`` fp32 [N, K, d, d] or None (zeros).  Returns the output in
    q's type and the final state: None, or ``final_state`` if that is a tensor (it may
    be initial_state, updated in place), or a new tensor if it is True.
    ``max_seqlen`` (ragged) is an upper bound of the lengths; it only chooses kernels."""
    shape = decay_shape(q, k, scale, cu_seqlens, max_seqlen)
    given = final_state if isinstance(final_state, torch.Tensor) else None
    _check_decay(q, k, v, log_decay, shape, ((initial_state, "initial_state"), (given, "final_state")))
    dev = q.device
    need = decay_workspace_bytes(shape, cu_seqlens is not None)
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        out = _like(out, "out", q)
        if given is None and final_state:
            d = shape.head_dim
            given = torch.empty((shape.batch, shape.kv_heads, d, d), dtype=torch.float32, device=dev)
        st = load_library().gbla_decay_forward(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(initial_state),
            _ptr(cu_seqlens), _ptr(workspace), workspace.numel(), _ptr(out), _ptr(given),
            _current(dev))
    _raise(st, "gbla_decay_forward")
    return out, given


def decay_attention_backward(q, k, v, log_decay, dout, scale: Optional[float] = None,
                             initial_state=None, dfinal_state=None, cu_seqlens=None,
                             max_seqlen=None, workspace=None, grads: Optional[dict] = None,
                             decay_grad: bool = True, stream=None) -> dict:
    """Gradients of sum(out * dout) + sum(final_state * dfinal_state) for the inputs of
    decay_attention: a dict with dq, dk, dv (in q's type), dlog_decay (fp32 [K]; left out
    with ``decay_grad`` False, for fixed decays) and, if initial_state is given,
    dinitial_state (fp32).  ``grads`` may hold outputs under
    those names; dinitial_state may be dfinal_state itself."""
    shape = decay_shape(q, k, scale, cu_seqlens, max_seqlen)
    g = dict(grads or {})
    _check_decay(q, k, v, log_decay, shape,
                 ((initial_state, "initial_state"), (dfinal_state, "dfinal_state"),
                  (g.get("dinitial_state"), "dinitial_state")))
    dev = q.device
    _want(dout, "dout", q.shape, q.dtype, dev)
    need = decay_backward_workspace_bytes(shape, cu_seqlens is not None)
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        g["dq"] = _like(g.get("dq"), "dq", q)
        g["dk"] = _like(g.get("dk"), "dk", k)
        g["dv"] = _like(g.get("dv"), "dv", k)
        if decay_grad:
            g["dlog_decay"] = _like(g.get("dlog_decay"), "dlog_decay", log_decay)
        if initial_state is not None and g.get("dinitial_state") is None:
            g["dinitial_state"] = torch.empty_like(initial_state)
        st = load_library().gbla_decay_backward(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(initial_state),
            _ptr(cu_seqlens), _ptr(dout), _ptr(dfinal_state), _ptr(workspace), workspace.numel(),
            _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]),
            _ptr(g["dlog_decay"]) if decay_grad else None, _ptr(g.get("dinitial_state")), _current(dev))
    _raise(st, "gbla_decay_backward")
    return g


def decay_step(q, k, v, log_decay, state, state_indices=None, scale: Optional[float] = None,
               out=None, stream=None) -> torch.Tensor:
    """decay_attention for one new token of each row: q [N, H, d], k, v [N, K, d],
    ``state`` fp32 [slots, K, d, d], updated in place.  Row n uses slot
    state_indices[n] (int32 [N]; without indices slot n).  Rows of one slot are applied
    in row order; a row whose index is outside the slots is skipped and its output row
    left as it is.  Returns the output [N, H, d] in q's type."""
    _check(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be [N, H, d]")
    N, H, d = q.shape
    dev, dtype = q.device, q.dtype
    K = _size_of(k, 3, 1)
    _want(k, "k", (N, K, d), dtype, dev)
    _want(v, "v", (N, K, d), dtype, dev)
    _want(log_decay, "log_decay", (K,), torch.float32, dev)
    slots = _size_of(state, 4, 0)
    _want(state, "state", (slots, K, d, d), torch.float32, dev)
    if state_indices is not None:
        _want(state_indices, "state_indices", (N,), torch.int32, dev)
    shape = DecayShape(N, 1, H, K, d, 0, _dtype_code(q), float(d) ** -0.5 if scale is None else float(scale))
    with _on(dev, stream):
        out = _like(out, "out", q)
        st = load_library().gbla_decay_step(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(state_indices),
            slots, _ptr(state), _ptr(out), _current(dev))
    _raise(st, "gbla_decay_step")
    return out


# ---------------------------------------------------------------------------
# The gated delta rule.
# ---------------------------------------------------------------------------
def delta_shape(q, k, v, scale: Optional[float] = None, cu_seqlens=None, max_seqlen=None) -> DeltaShape:
    B, n, H, K, d = _query_key(q, k, cu_seqlens)
    if K != H:
        raise ValueError("k must have as many heads as q")
    V = _size_of(v, 4, 1) if cu_seqlens is None else _size_of(v, 3, 0)
    _want(v, "v", (B, V, n, d) if cu_seqlens is None else (V, n, d), q.dtype, q.device)
    msl = 0
    if cu_seqlens is not None:
        msl = int(max_seqlen) if max_seqlen is not None else n
    return DeltaShape(B, n, H, V, d, msl, _dtype_code(q),
                      float(d) ** -0.5 if scale is None else float(scale))


def delta_workspace_bytes(shape: DeltaShape, ragged: bool = False) -> int:
    """``ragged``: for calls with cu_seqlens only, which take less than both readings."""
    return _scratch("gbla_delta", shape, ragged)


def delta_backward_workspace_bytes(shape: DeltaShape, ragged: bool = False) -> int:
    return _scratch("gbla_delta_backward", shape, ragged)


def _check_delta(v, log_decay, beta, shape, states):
    dev = v.device
    _want(log_decay, "log_decay", v.shape[:-1], torch.float32, dev)
    _want(beta, "beta", v.shape[:-1], torch.float32, dev)
    for t, name in states:
        if t is not None:
            _want(t, name, (shape.batch, shape.value_heads, shape.head_dim, shape.head_dim),
                  torch.float32, dev)


def delta_attention(q, k, v, log_decay, beta, scale: Optional[float] = None, initial_state=None,
                    final_state=None, cu_seqlens=None, max_seqlen=None, workspace=None, out=None,
                    stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """The gated delta rule, u_t = beta_t (v_t - exp(g_t) S_{t-1}^T k_t), S_t = exp(g_t) S_{t-1}
    + k_t u_t^T, o_t = scale S_t^T q_t (scale d^-1/2 by default); see include/gbla.h.
    q, k [B, H, n, d] or [H, T, d]; v with V heads, H dividing V; log_decay (<= 0) and beta
    fp32 [B, V, n] or [V, T]; ``initial_state`` fp32 [N, V, d, d] or None (zeros).  Returns the
    output, like v, and the final state: None, or ``final_state`` if that is a tensor (it may be
    initial_state, updated in place), or a new tensor if it is True.
    ``max_seqlen`` (ragged) is an upper bound of the lengths; it only chooses kernels."""
    shape = delta_shape(q, k, v, scale, cu_seqlens, max_seqlen)
    given = final_state if isinstance(final_state, torch.Tensor) else None
    _check_delta(v, log_decay, beta, shape, ((initial_state, "initial_state"), (given, "final_state")))
    dev = q.device
    need = delta_workspace_bytes(shape, cu_seqlens is not None)
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        out = _like(out, "out", v)
        if given is None and final_state:
            d = shape.head_dim
            given = torch.empty((shape.batch, shape.value_heads, d, d), dtype=torch.float32, device=dev)
        st = load_library().gbla_delta_forward(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(beta),
            _ptr(initial_state), _ptr(cu_seqlens), _ptr(workspace), workspace.numel(), _ptr(out),
            _ptr(given), _current(dev))
    _raise(st, "gbla_delta_forward")
    return out, given


def delta_attention_backward(q, k, v, log_decay, beta, dout, scale: Optional[float] = None,
                             initial_state=None, dfinal_state=None, cu_seqlens=None, max_seqlen=None,
                             workspace=None, grads: Optional[dict] = None, stream=None) -> dict:
    """Gradients of sum(out * dout) + sum(final_state * dfinal_state) for the inputs of
    delta_attention: a dict with dq, dk, dv (in q's type), dlog_decay, dbeta (fp32) and, if
    initial_state is given, dinitial_state (fp32).  ``grads`` may hold outputs under those
    names; dinitial_state may be dfinal_state itself."""
    shape = delta_shape(q, k, v, scale, cu_seqlens, max_seqlen)
    g = dict(grads or {})
    _check_delta(v, log_decay, beta, shape,
                 ((initial_state, "initial_state"), (dfinal_state, "dfinal_state"),
                  (g.get("dinitial_state"), "dinitial_state")))
    dev = q.device
    _want(dout, "dout", v.shape, q.dtype, dev)
    need = delta_backward_workspace_bytes(shape, cu_seqlens is not None)
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        for name, like in (("dq", q), ("dk", k), ("dv", v), ("dlog_decay", log_decay), ("dbeta", beta)):
            g[name] = _like(g.get(name), name, like)
        if initial_state is not None and g.get("dinitial_state") is None:
            g["dinitial_state"] = torch.empty_like(initial_state)
        st = load_library().gbla_delta_backward(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(beta),
            _ptr(initial_state), _ptr(cu_seqlens), _ptr(dout), _ptr(dfinal_state), _ptr(workspace),
            workspace.numel(), _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]), _ptr(g["dlog_decay"]),
            _ptr(g["dbeta"]), _ptr(g.get("dinitial_state")), _current(dev))
    _raise(st, "gbla_delta_backward")
    return g


def delta_step(q, k, v, log_decay, beta, state, state_indices=None, scale: Optional[float] = None,
               out=None, stream=None) -> torch.Tensor:
    """delta_attention for one new token of each row: q, k [N, H, d], v [N, V, d], log_decay and
    beta fp32 [N, V], ``state`` fp32 [slots, V, d, d], updated in place.  Row n uses slot
    state_indices[n] (int32 [N]; without indices slot n).  Rows of one slot are applied in row
    order; a row whose index is outside the slots is skipped and its output row left as it is.
    Returns the output, like v."""
    _check(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be [N, H, d]")
    N, H, d = q.shape
    dev, dtype = q.device, q.dtype
    V = _size_of(v, 3, 1)
    _want(k, "k", q.shape, dtype, dev)
    _want(v, "v", (N, V, d), dtype, dev)
    _want(log_decay, "log_decay", (N, V), torch.float32, dev)
    _want(beta, "beta", (N, V), torch.float32, dev)
    slots = _size_of(state, 4, 0)
    _want(state, "state", (slots, V, d, d), torch.float32, dev)
    if state_indices is not None:
        _want(state_indices, "state_indices", (N,), torch.int32, dev)
    shape = DeltaShape(N, 1, H, V, d, 0, _dtype_code(q), float(d) ** -0.5 if scale is None else float(scale))
    with _on(dev, stream):
        out = _like(out, "out", v)
        st = load_library().gbla_delta_step(
            ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(beta),
            _ptr(state_indices), slots, _ptr(state), _ptr(out), _current(dev))
    _raise(st, "gbla_delta_step")
    return out


# ---------------------------------------------------------------------------
# The residual stream's norm.
# ---------------------------------------------------------------------------
def norm_shape(x, eps: float = 1e-6, out_dtype: Optional[int] = None, group: int = 0) -> NormShape:
    _check(x, "x")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be [..., width]")
    width = x.shape[-1]
    code = _dtype_code(x)
    return NormShape(x.numel() // width, width, code, code if out_dtype is None else out_dtype, int(group),
                     float(eps))


def _add_norm(shape, x, weight, residual, total, out, scales, stream):
    dev = x.device
    _want(weight, "weight", (shape.width,), torch.float32, dev)
    if residual is not None:
        _want(residual, "residual", x.shape, x.dtype, dev)
    if total is not None:
        _want(total, "sum_out", x.shape, x.dtype, dev)
    with _on(dev, stream):
        if total is None:
            total = x if residual is None else torch.empty_like(x)
        if shape.out_dtype == GBLA_E4M3:
            each = shape.group or shape.width
            if out is None:
                out = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=dev)
            if scales is None:
                scales = torch.empty(x.shape[:-1] + (shape.width // each,), dtype=torch.float32, device=dev)
            _want(out, "out", x.shape, torch.float8_e4m3fn, dev)
            _want(scales, "scales", x.shape[:-1] + (shape.width // each,), torch.float32, dev)
        else:
            out = _like(out, "out", x)
        st = load_library().gbla_add_norm(
            ctypes.byref(shape), _ptr(x), _ptr(residual), _ptr(weight),
            None if total is x and residual is None else _ptr(total), _ptr(out), _ptr(scales), _current(dev))
    _raise(st, "gbla_add_norm")
    return out, scales, total


def add_rms_norm(x, weight, residual=None, eps: float = 1e-6, sum_out=None, out=None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """s = x + residual in x's type (x if residual is None) and y = s / sqrt(mean s^2 + eps) *
    weight over the last dimension, in x's type; see include/gbla.h.  x [..., width], weight fp32
    [width].  Returns (y, s); s is x itself without a residual.  ``sum_out`` and ``out`` may be x
    or residual themselves, not both the same one."""
    shape = norm_shape(x, eps)
    out, _, total = _add_norm(shape, x, weight, residual, sum_out, out, None, stream)
    return out, total


def add_rms_norm_e4m3(x, weight, residual=None, eps: float = 1e-6, group: int = 0, sum_out=None, out=None,
                      scales=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """add_rms_norm with y in eight bits: returns (y as float8_e4m3fn, scales, s), where y stands
    for out * scale.  ``group`` 128: a scale for every 128 channels (fp32 [..., width / 128]),
    0: one a row ([..., 1])."""
    shape = norm_shape(x, eps, GBLA_E4M3, group)
    return _add_norm(shape, x, weight, residual, sum_out, out, scales, stream)


def add_rms_norm_backward_workspace_bytes(shape: NormShape) -> int:
    n = load_library().gbla_add_norm_backward_workspace_bytes(ctypes.byref(shape))
    if n == 0:
        raise GblaError(1, "gbla_add_norm_backward_workspace_bytes")
    return int(n)


def add_rms_norm_backward(total, weight, dout, dsum=None, eps: float = 1e-6, workspace=None,
                          grads: Optional[dict] = None, stream=None) -> dict:
    """Gradients of sum(y * dout) + sum(s * dsum), from the s that add_rms_norm returned: a dict
    with dx (of x and of residual alike, in x's type) and dweight (fp32).  ``dsum`` None: zeros.
    ``grads`` may hold outputs under those names; dx may be dout or dsum itself."""
    shape = norm_shape(total, eps)
    dev = total.device
    _want(weight, "weight", (shape.width,), torch.float32, dev)
    _want(dout, "dout", total.shape, total.dtype, dev)
    if dsum is not None:
        _want(dsum, "dsum", total.shape, total.dtype, dev)
    need = add_rms_norm_backward_workspace_bytes(shape)
    g = dict(grads or {})
    with _on(dev, stream):
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check_ws(workspace, dev, need)
        g["dx"] = _like(g.get("dx"), "dx", total)
        g["dweight"] = _like(g.get("dweight"), "dweight", weight)
        st = load_library().gbla_add_norm_backward(
            ctypes.byref(shape), _ptr(total), _ptr(weight), _ptr(dout), _ptr(dsum), _ptr(workspace),
            workspace.numel(), _ptr(g["dx"]), _ptr(g["dweight"]), _current(dev))
    _raise(st, "gbla_add_norm_backward")
    return g
