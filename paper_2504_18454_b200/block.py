"""ctypes binding of include/palsgd_block.h over torch tensors: the operators with which K workers make their gradients.

Every call takes tensors whose first axis is the worker; a worker's weights may lie anywhere at a constant stride (a
view of the rows of a packed ReplicaArena: `ReplicaArena.worker_tensor`).  The last axis is contiguous.  `stream` is a
raw cudaStream_t; None is torch's current stream of the tensors' device.  Outputs and workspaces that the caller does
not give are allocated for that stream.  Calls are asynchronous.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import NamedTuple, Optional, Tuple, Union

import torch

from .binding import PREC_BF16_MASTER, PREC_FP32, PalsgdError
from .binding import lib as _base_lib

ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2, 3
SAVE_NONE, SAVE_FULL, SAVE_8BIT = 0, 1, 2
ACT8_GROUP = 32
EINVAL = -1


class Mat(C.Structure):
    _fields_ = [("data", C.c_void_p), ("worker_stride", C.c_int64), ("row_stride", C.c_int64)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("worker_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64)]


class FfnShape(C.Structure):
    _fields_ = [("K", C.c_uint32), ("precision", C.c_int32), ("activation", C.c_int32), ("save", C.c_int32),
                ("tokens", C.c_uint64), ("d_model", C.c_uint64), ("d_ff", C.c_uint64)]


class QkShape(C.Structure):
    _fields_ = [("K", C.c_uint32), ("precision", C.c_int32), ("tokens", C.c_uint64), ("heads_q", C.c_uint32),
                ("heads_k", C.c_uint32), ("head_dim", C.c_uint32), ("rotary_dim", C.c_uint32),
                ("interleaved", C.c_int32), ("reserved_", C.c_uint32), ("table_rows", C.c_uint64),
                ("pos_worker_stride", C.c_int64), ("eps", C.c_double)]


class Act8(NamedTuple):
    """An 8-bit activation checkpoint: q * 2^(exponent - 127), one exponent per 32 values of the last axis."""
    q: torch.Tensor              # int8 (K, rows, cols) or (rows, cols)
    exponent: torch.Tensor       # uint8 (..., rows, ceil(cols / 32))
    dtype: torch.dtype           # what it was taken from


Saved = Union[torch.Tensor, Act8]
_ready = False


def lib() -> C.CDLL:
    global _ready
    L = _base_lib()
    if not _ready:
        vp, u32, u64, i32, M, H = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int32, C.POINTER(Mat), C.POINTER(Heads)
        size = C.POINTER(C.c_size_t)
        L.palsgd_act8_pack.argtypes = L.palsgd_act8_unpack.argtypes = [i32, u32, u64, u64, M, M, M, vp]
        L.palsgd_ffn_forward.argtypes = [C.POINTER(FfnShape)] + [M] * 9 + [vp, size, vp]
        L.palsgd_ffn_backward.argtypes = [C.POINTER(FfnShape)] + [M] * 14 + [vp, size, vp]
        L.palsgd_qk_norm_rope_forward.argtypes = [C.POINTER(QkShape), H, H, M, M, vp, vp, vp, H, H, vp]
        L.palsgd_qk_norm_rope_backward.argtypes = ([C.POINTER(QkShape), H, H, H, H, M, M, vp, vp, vp, H, H, M, M]
                                                   + [vp, size, vp])
        L.palsgd_block_status.argtypes = [vp]
        for n in ("block_status", "act8_pack", "act8_unpack", "ffn_forward", "ffn_backward", "qk_norm_rope_forward",
                  "qk_norm_rope_backward"):
            getattr(L, "palsgd_" + n).restype = C.c_int
        _ready = True
    return L


# ---------------------------------------------------------------------------------------------- argument marshalling

def _refuse(where: str, why: str):
    raise PalsgdError(EINVAL, where, why)


def _check(rc: int, where: str) -> None:
    if rc:
        raise PalsgdError(rc, where, lib().palsgd_last_cuda_error(None).decode() if rc == -3 else "")


def _precision(t: torch.Tensor, where: str, name: str) -> int:
    if t.dtype == torch.float32:
        return PREC_FP32
    if t.dtype == torch.bfloat16:
        return PREC_BF16_MASTER
    _refuse(where, f"{name} must be float32 or bfloat16, not {t.dtype}")


def _tensor(t, where: str, name: str, shape, dtype, device) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        _refuse(where, f"{name} must be a tensor")
    if tuple(t.shape) != tuple(shape):
        _refuse(where, f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype:
        _refuse(where, f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        _refuse(where, f"{name} must be on {device}, not {t.device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
        _refuse(where, f"the last axis of {name} must be contiguous")
    return t


def _cuda(t, where: str, name: str, ndim: int) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(where, f"{name} must be a CUDA tensor")
    if t.dim() != ndim:
        _refuse(where, f"{name} must have {ndim} axes, not {t.dim()}")
    return t.device


def _mat(t: Optional[torch.Tensor]):
    """(K, rows, cols) or (K, cols) -> palsgd_mat*; strides of axes of length <= 1 do not matter and become 0."""
    if t is None:
        return None
    s = [st if n > 1 else 0 for n, st in zip(t.shape, t.stride())]
    return C.byref(Mat(t.data_ptr(), s[0], s[1] if t.dim() == 3 else 0))


def _heads(t: torch.Tensor):
    s = [st if n > 1 else 0 for n, st in zip(t.shape, t.stride())]
    return C.byref(Heads(t.data_ptr(), s[0], s[1], s[2]))


class _On:
    """The device and the stream of a call: `raw` is the cudaStream_t; allocations inside the block belong to it."""

    def __init__(self, device: torch.device, stream: Optional[int]):
        self.device, self.stream = device, stream
        self.stack = None

    def __enter__(self) -> "_On":
        current = torch.cuda.current_stream(self.device).cuda_stream
        self.raw = C.c_void_p(current if self.stream is None else self.stream)
        if torch.cuda.current_device() != self.device.index or (self.stream is not None and self.stream != current):
            self.stack = contextlib.ExitStack()
            self.stack.enter_context(torch.cuda.device(self.device))
            if self.stream is not None and self.stream != current:
                # stream 0 is the legacy default stream, which torch knows as its default stream
                self.stack.enter_context(torch.cuda.stream(
                    torch.cuda.ExternalStream(self.stream, self.device) if self.stream
                    else torch.cuda.default_stream(self.device)))
        return self

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()


def _workspace(call, given: Optional[torch.Tensor], device, where: str):
    """call(workspace pointer, bytes pointer) twice: for the size, then with the memory."""
    n = C.c_size_t(0)
    _check(call(None, C.byref(n)), where)
    if given is None:
        given = torch.empty(max(n.value, 1), dtype=torch.uint8, device=device)
    elif given.dtype != torch.uint8 or given.device != device or not given.is_contiguous():
        _refuse(where, f"workspace must be a contiguous uint8 tensor on {device}")
    n.value = given.numel()
    _check(call(C.c_void_p(given.data_ptr()), C.byref(n)), where)


def block_status(stream: Optional[int] = None) -> None:
    """palsgd_block_status: raises PalsgdError if a matrix kernel's bounded wait gave up since the last call (its outputs
    are then unspecified).  Synchronises the stream."""
    raw = torch.cuda.current_stream().cuda_stream if stream is None else stream
    _check(lib().palsgd_block_status(C.c_void_p(raw)), "palsgd_block_status")


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints

def _three(t: torch.Tensor) -> torch.Tensor:
    return t[None] if t.dim() == 2 else t


def act8_pack(x: torch.Tensor, *, out: Optional[Act8] = None, stream: Optional[int] = None) -> Act8:
    """palsgd_act8_pack: the 8-bit checkpoint of x (rows, cols) or (K, rows, cols), float32 or bfloat16."""
    where = "palsgd_act8_pack"
    dev = _cuda(x, where, "x", 2 if isinstance(x, torch.Tensor) and x.dim() == 2 else 3)
    prec = _precision(x, where, "x")
    _tensor(x, where, "x", x.shape, x.dtype, dev)
    groups = (x.shape[-1] + ACT8_GROUP - 1) // ACT8_GROUP
    with _On(dev, stream) as on:
        if out is None:
            out = Act8(torch.empty(x.shape, dtype=torch.int8, device=dev),
                       torch.empty(*x.shape[:-1], groups, dtype=torch.uint8, device=dev), x.dtype)
        else:
            _tensor(out.q, where, "out.q", x.shape, torch.int8, dev)
            _tensor(out.exponent, where, "out.exponent", (*x.shape[:-1], groups), torch.uint8, dev)
        v = _three(x)
        _check(lib().palsgd_act8_pack(prec, v.shape[0], v.shape[1], v.shape[2], _mat(v), _mat(_three(out.q)),
                                      _mat(_three(out.exponent)), on.raw), where)
    return out


def act8_unpack(a: Act8, *, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                stream: Optional[int] = None) -> torch.Tensor:
    """palsgd_act8_unpack: the values that a checkpoint stands for, in `dtype` (default: the type it was taken from).
    They have at most eight significant bits: bfloat16 holds them exactly."""
    where = "palsgd_act8_unpack"
    dev = _cuda(a.q, where, "q", 2 if isinstance(a.q, torch.Tensor) and a.q.dim() == 2 else 3)
    _tensor(a.q, where, "q", a.q.shape, torch.int8, dev)
    _tensor(a.exponent, where, "exponent", (*a.q.shape[:-1], (a.q.shape[-1] + ACT8_GROUP - 1) // ACT8_GROUP),
            torch.uint8, dev)
    dtype = dtype or (out.dtype if out is not None else a.dtype)
    with _On(dev, stream) as on:
        if out is None:
            out = torch.empty(a.q.shape, dtype=dtype, device=dev)
        prec = _precision(out, where, "out")
        _tensor(out, where, "out", a.q.shape, dtype, dev)
        v = _three(out)
        _check(lib().palsgd_act8_unpack(prec, v.shape[0], v.shape[1], v.shape[2], _mat(_three(a.q)),
                                        _mat(_three(a.exponent)), _mat(v), on.raw), where)
    return out


# ---------------------------------------------------------------------------------------------- gated feed-forward

def _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev):
    F = w_gate.shape[1] if isinstance(w_gate, torch.Tensor) and w_gate.dim() == 3 else 0
    _tensor(w_gate, where, "w_gate", (K, F, D), dt, dev)
    _tensor(w_up, where, "w_up", (K, F, D), dt, dev)
    _tensor(w_down, where, "w_down", (K, D, F), dt, dev)
    return F


def _act8_args(where, a: Act8, name, shape, dev):
    _tensor(a.q, where, name + ".q", shape, torch.int8, dev)
    _tensor(a.exponent, where, name + ".exponent", (*shape[:-1], (shape[-1] + ACT8_GROUP - 1) // ACT8_GROUP),
            torch.uint8, dev)


def ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, *,
                activation: int = ACT_SILU, save: int = SAVE_FULL, out: Optional[torch.Tensor] = None,
                saved: Optional[Tuple[Saved, Saved]] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[int] = None) -> Tuple[torch.Tensor, Optional[Tuple[Saved, Saved]]]:
    """palsgd_ffn_forward: y = (act(x w_gate^T) * (x w_up^T)) w_down^T for K workers.

    x (K, tokens, d_model), w_gate and w_up (K, d_ff, d_model), w_down (K, d_model, d_ff).  Returns y and what
    `ffn_backward` needs besides its arguments: (gate, up) as tensors, as Act8, or None, by `save`.  `out`, `saved` and
    `workspace` give the memory to write to.
    """
    where = "palsgd_ffn_forward"
    dev = _cuda(x, where, "x", 3)
    prec, dt = _precision(x, where, "x"), x.dtype
    K, M, D = x.shape
    _tensor(x, where, "x", x.shape, dt, dev)
    F = _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev)
    shape = FfnShape(K, prec, int(activation), int(save), M, D, F)
    with _On(dev, stream) as on:
        y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else _tensor(out, where, "out", x.shape, dt, dev)
        if save == SAVE_NONE:
            saved = None
        elif saved is None:
            if save == SAVE_8BIT:
                G = (F + ACT8_GROUP - 1) // ACT8_GROUP
                saved = tuple(Act8(torch.empty(K, M, F, dtype=torch.int8, device=dev),
                                   torch.empty(K, M, G, dtype=torch.uint8, device=dev), dt) for _ in range(2))
            else:
                saved = tuple(torch.empty(K, M, F, dtype=dt, device=dev) for _ in range(2))
        mats = _saved_mats(where, save, saved, (K, M, F), dt, dev)
        call = lambda ws, n: lib().palsgd_ffn_forward(
            C.byref(shape), _mat(x), _mat(w_gate), _mat(w_up), _mat(w_down), _mat(y), *mats, ws, n, on.raw)
        _workspace(call, workspace, dev, where)
    return y, saved


def _saved_mats(where, save, saved, shape, dt, dev):
    """gate, up, gate_e, up_e as palsgd_mat*"""
    if save == SAVE_NONE:
        return None, None, None, None
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    gate, up = saved
    if save == SAVE_8BIT:
        if not (isinstance(gate, Act8) and isinstance(up, Act8)):
            _refuse(where, "gate and up must both be Act8")
        _act8_args(where, gate, "gate", shape, dev)
        _act8_args(where, up, "up", shape, dev)
        return _mat(gate.q), _mat(up.q), _mat(gate.exponent), _mat(up.exponent)
    _tensor(gate, where, "gate", shape, dt, dev)
    _tensor(up, where, "up", shape, dt, dev)
    return _mat(gate), _mat(up), None, None


def ffn_backward(dy: torch.Tensor, x: Saved, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                 saved: Tuple[Saved, Saved], *, activation: int = ACT_SILU, need_dx: bool = True,
                 out: Optional[Tuple] = None, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[int] = None):
    """palsgd_ffn_backward: (dx, dw_gate, dw_up, dw_down) from dy and what the forward call saved.

    With (gate, up) as Act8, x may be an Act8 too.  `out` = (dx, dw_gate, dw_up, dw_down) gives the memory to write to
    (e.g. the workers' gradient buffers); entries may be None.  need_dx = False leaves dx out (it comes back as None).
    """
    where = "palsgd_ffn_backward"
    dev = _cuda(dy, where, "dy", 3)
    prec, dt = _precision(dy, where, "dy"), dy.dtype
    K, M, D = dy.shape
    _tensor(dy, where, "dy", dy.shape, dt, dev)
    F = _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev)
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    save = SAVE_8BIT if isinstance(saved[0], Act8) else SAVE_FULL
    if isinstance(x, Act8):
        _act8_args(where, x, "x", (K, M, D), dev)
        if save != SAVE_8BIT:
            _refuse(where, "x may be an Act8 only where gate and up are")
        mx, mxe = _mat(x.q), _mat(x.exponent)
    else:
        _tensor(x, where, "x", (K, M, D), dt, dev)
        mx, mxe = _mat(x), None
    shape = FfnShape(K, prec, int(activation), save, M, D, F)
    with _On(dev, stream) as on:
        want = ((K, M, D), (K, F, D), (K, F, D), (K, D, F))
        outs = list(out) if out is not None else [None] * 4
        if len(outs) != 4:
            _refuse(where, "out must be (dx, dw_gate, dw_up, dw_down)")
        for i, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
            if i == 0 and not need_dx:
                outs[0] = None
            elif outs[i] is None:
                outs[i] = torch.empty(want[i], dtype=dt, device=dev)
            else:
                _tensor(outs[i], where, name, want[i], dt, dev)
        mats = _saved_mats(where, save, saved, (K, M, F), dt, dev)
        call = lambda ws, n: lib().palsgd_ffn_backward(
            C.byref(shape), _mat(dy), mx, mxe, _mat(w_gate), _mat(w_up), _mat(w_down), *mats,
            *(_mat(t) for t in outs), ws, n, on.raw)
        _workspace(call, workspace, dev, where)
    return tuple(outs)


# ---------------------------------------------------------------------------------------------- q/k norm + rotation

def _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved):
    dev = _cuda(q, where, "q", 4)
    prec, dt = _precision(q, where, "q"), q.dtype
    K, M, HQ, DH = q.shape
    HK = k.shape[2] if isinstance(k, torch.Tensor) and k.dim() == 4 else -1
    _tensor(q, where, "q", q.shape, dt, dev)
    _tensor(k, where, "k", (K, M, HK, DH), dt, dev)
    _tensor(w_q, where, "w_q", (K, DH), dt, dev)
    _tensor(w_k, where, "w_k", (K, DH), dt, dev)
    if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
        _refuse(where, "cos must be a (rows, rotary_dim / 2) tensor")
    for name, t in (("cos", cos), ("sin", sin)):
        if not _tensor(t, where, name, cos.shape, torch.float32, dev).is_contiguous():
            _refuse(where, f"{name} must be contiguous")
    _tensor(positions, where, "positions", (K, M), torch.int32, dev)
    shape = QkShape(K, prec, M, HQ, HK, DH, 2 * cos.shape[1], int(bool(interleaved)), 0, cos.shape[0],
                    positions.stride(0) if K > 1 else 0, float(eps))
    vp = C.c_void_p
    return dev, shape, (vp(cos.data_ptr()), vp(sin.data_ptr()), vp(positions.data_ptr()))


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[int] = None):
    """palsgd_qk_norm_rope_forward: RMS norm of every head of q (K, tokens, heads_q, head_dim) and k, with weights
    w_q, w_k (K, head_dim), then the rotation of the first 2*cos.shape[1] values by the angle tables cos, sin
    (rows, rotary_dim / 2) at positions (K, tokens) int32.  Returns (q_out, k_out)."""
    where = "palsgd_qk_norm_rope_forward"
    dev, shape, tables = _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    with _On(dev, stream) as on:
        if out is None:
            out = tuple(torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k))
        else:
            _tensor(out[0], where, "q_out", q.shape, q.dtype, dev)
            _tensor(out[1], where, "k_out", k.shape, q.dtype, dev)
        _check(lib().palsgd_qk_norm_rope_forward(C.byref(shape), _heads(q), _heads(k), _mat(w_q), _mat(w_k), *tables,
                                                 _heads(out[0]), _heads(out[1]), on.raw), where)
    return tuple(out)


def qk_norm_rope_backward(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
                          positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                          out: Optional[Tuple] = None, workspace: Optional[torch.Tensor] = None,
                          stream: Optional[int] = None):
    """palsgd_qk_norm_rope_backward: (dq, dk, dw_q, dw_k) from the gradients of qk_norm_rope's results and its inputs.
    `out` gives the memory to write to; entries may be None."""
    where = "palsgd_qk_norm_rope_backward"
    dev, shape, tables = _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    _tensor(dq_out, where, "dq_out", q.shape, q.dtype, dev)
    _tensor(dk_out, where, "dk_out", k.shape, q.dtype, dev)
    with _On(dev, stream) as on:
        outs = list(out) if out is not None else [None] * 4
        if len(outs) != 4:
            _refuse(where, "out must be (dq, dk, dw_q, dw_k)")
        for i, (name, like) in enumerate((("dq", q), ("dk", k), ("dw_q", w_q), ("dw_k", w_k))):
            if outs[i] is None:
                outs[i] = torch.empty(like.shape, dtype=q.dtype, device=dev)
            else:
                _tensor(outs[i], where, name, like.shape, q.dtype, dev)
        call = lambda ws, n: lib().palsgd_qk_norm_rope_backward(
            C.byref(shape), _heads(dq_out), _heads(dk_out), _heads(q), _heads(k), _mat(w_q), _mat(w_k), *tables,
            _heads(outs[0]), _heads(outs[1]), _mat(outs[2]), _mat(outs[3]), ws, n, on.raw)
        _workspace(call, workspace, dev, where)
    return tuple(outs)
