"""Binding of include/palsgd_block.h over torch tensors: the operators with which K workers make their gradients.

Every call takes tensors whose first axis is the worker; a worker's weights may lie anywhere at a constant stride (a
view of the rows of a packed ReplicaArena: `ReplicaArena.worker_tensor`).  The last axis is contiguous.  `stream` is a
raw cudaStream_t; None is torch's current stream of the tensors' device.  Outputs and workspaces that the caller does
not give are allocated for that stream; inputs that belong to another stream have to outlive the call there
(`Tensor.record_stream`), as with torch's own operators.  Calls are asynchronous.  Arguments are checked and packed by the
native module `_block` (csrc/block_torch.cpp); a refused one raises PalsgdError: outputs that overlap an input among them, but
for a head matrix that the q/k operator writes in place.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Tuple, Union

import torch

from .binding import PalsgdError
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
_native = None


def lib() -> C.CDLL:
    """libpalsgd.so with the argument types of palsgd_block.h (struct pointers as plain addresses)."""
    global _ready
    L = _base_lib()
    if not _ready:
        vp, u32, u64, i32 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int32
        L.palsgd_act8_pack.argtypes = L.palsgd_act8_unpack.argtypes = [i32, u32, u64, u64] + [vp] * 4
        for n, args in (("ffn_forward", 13), ("ffn_backward", 18), ("qk_norm_rope_forward", 11),
                        ("qk_norm_rope_backward", 17), ("block_status", 1)):
            getattr(L, "palsgd_" + n).argtypes = [vp] * args
        for n in ("block_status", "act8_pack", "act8_unpack", "ffn_forward", "ffn_backward", "qk_norm_rope_forward",
                  "qk_norm_rope_backward"):
            getattr(L, "palsgd_" + n).restype = C.c_int
        _ready = True
    return L


def _ext():
    """The native module, bound to the loaded library.  There is no fallback: a missing one is an error."""
    global _native
    if _native is None:
        L = lib()
        try:
            from . import _block
        except ImportError as e:
            raise ImportError("paper_2504_18454_b200/_block.so is missing or does not fit the installed torch: build it with "
                              "`python -m paper_2504_18454_b200.build`") from e
        _block.bind(L._handle, PalsgdError)
        _native = _block
    return _native


def _refuse(where: str, why: str):
    raise PalsgdError(EINVAL, where, why)


def block_status(stream: Optional[int] = None) -> None:
    """palsgd_block_status: raises PalsgdError if a matrix kernel's bounded wait gave up since the last call (its outputs
    are then unspecified).  Synchronises the stream."""
    raw = torch.cuda.current_stream().cuda_stream if stream is None else stream
    rc = lib().palsgd_block_status(C.c_void_p(raw))
    if rc:
        raise PalsgdError(rc, "palsgd_block_status", lib().palsgd_last_cuda_error(None).decode() if rc == -3 else "")


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints

def act8_pack(x: torch.Tensor, *, out: Optional[Act8] = None, stream: Optional[int] = None) -> Act8:
    """palsgd_act8_pack: the 8-bit checkpoint of x (rows, cols) or (K, rows, cols), float32 or bfloat16."""
    native = _native or _ext()
    if out is None:
        return Act8(*native.act8_pack(x, None, None, stream), x.dtype)
    native.act8_pack(x, out.q, out.exponent, stream)
    return out


def act8_unpack(a: Act8, *, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                stream: Optional[int] = None) -> torch.Tensor:
    """palsgd_act8_unpack: the values that a checkpoint stands for, in `dtype` (default: the type it was taken from).
    They have at most eight significant bits: bfloat16 holds them exactly."""
    native = _native or _ext()
    return native.act8_unpack(a.q, a.exponent, dtype or (a.dtype if out is None else out.dtype), out, stream)


# ---------------------------------------------------------------------------------------------- gated feed-forward

def _saved(where: str, save: int, saved):
    """gate, up and their exponents, or None."""
    if saved is None or save == SAVE_NONE:
        return None, None, None, None
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    gate, up = saved
    if save == SAVE_8BIT:
        if not (isinstance(gate, Act8) and isinstance(up, Act8)):
            _refuse(where, "gate and up must both be Act8")
        return gate.q, up.q, gate.exponent, up.exponent
    return gate, up, None, None


def ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, *,
                activation: int = ACT_SILU, save: int = SAVE_FULL, out: Optional[torch.Tensor] = None,
                saved: Optional[Tuple[Saved, Saved]] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[int] = None) -> Tuple[torch.Tensor, Optional[Tuple[Saved, Saved]]]:
    """palsgd_ffn_forward: y = (act(x w_gate^T) * (x w_up^T)) w_down^T for K workers.

    x (K, tokens, d_model), w_gate and w_up (K, d_ff, d_model), w_down (K, d_model, d_ff).  Returns y and what
    `ffn_backward` needs besides its arguments: (gate, up) as tensors, as Act8, or None, by `save`.  `out`, `saved` and
    `workspace` give the memory to write to.
    """
    native = _native or _ext()
    y, gate, up, gate_e, up_e = native.ffn_forward(
        x, w_gate, w_up, w_down, activation, save, out, *_saved("palsgd_ffn_forward", save, saved), workspace, stream)
    if save == SAVE_8BIT:
        return y, (Act8(gate, gate_e, x.dtype), Act8(up, up_e, x.dtype))
    return y, None if save == SAVE_NONE else (gate, up)


def ffn_backward(dy: torch.Tensor, x: Saved, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                 saved: Tuple[Saved, Saved], *, activation: int = ACT_SILU, need_dx: bool = True,
                 out: Optional[Tuple] = None, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[int] = None):
    """palsgd_ffn_backward: (dx, dw_gate, dw_up, dw_down) from dy and what the forward call saved.

    With (gate, up) as Act8, x may be an Act8 too.  `out` = (dx, dw_gate, dw_up, dw_down) gives the memory to write to
    (e.g. the workers' gradient buffers); entries may be None.  need_dx = False leaves dx out (it comes back as None).
    """
    where = "palsgd_ffn_backward"
    native = _native or _ext()
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    save = SAVE_8BIT if isinstance(saved[0], Act8) else SAVE_FULL
    x_e = None
    if isinstance(x, Act8):
        if save != SAVE_8BIT:
            _refuse(where, "x may be an Act8 only where gate and up are")
        x, x_e = x.q, x.exponent
    out = (None,) * 4 if out is None else out
    if len(out) != 4:
        _refuse(where, "out must be (dx, dw_gate, dw_up, dw_down)")
    return native.ffn_backward(dy, x, x_e, w_gate, w_up, w_down, activation, save, *_saved(where, save, saved),
                               1 if need_dx else 0, *out, workspace, stream)


# ---------------------------------------------------------------------------------------------- q/k norm + rotation

def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[int] = None):
    """palsgd_qk_norm_rope_forward: RMS norm of every head of q (K, tokens, heads_q, head_dim) and k, with weights
    w_q, w_k (K, head_dim), then the rotation of the first 2*cos.shape[1] values by the angle tables cos, sin
    (rows, rotary_dim / 2) at positions (K, tokens) int32.  Returns (q_out, k_out)."""
    native = _native or _ext()
    oq, ok = (None, None) if out is None else out
    return native.qk_forward(q, k, w_q, w_k, cos, sin, positions, eps, 1 if interleaved else 0, oq, ok, stream)


def qk_norm_rope_backward(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
                          positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                          out: Optional[Tuple] = None, workspace: Optional[torch.Tensor] = None,
                          stream: Optional[int] = None):
    """palsgd_qk_norm_rope_backward: (dq, dk, dw_q, dw_k) from the gradients of qk_norm_rope's results and its inputs.
    `out` gives the memory to write to; entries may be None."""
    native = _native or _ext()
    out = (None,) * 4 if out is None else out
    if len(out) != 4:
        _refuse("palsgd_qk_norm_rope_backward", "out must be (dq, dk, dw_q, dw_k)")
    return native.qk_backward(q, k, w_q, w_k, cos, sin, positions, eps, 1 if interleaved else 0, dq_out, dk_out, *out,
                              workspace, stream)
