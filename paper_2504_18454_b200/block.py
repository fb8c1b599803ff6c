"""ctypes binding of include/palsgd_block.h over torch tensors: the operators with which K workers make their gradients.

Every call takes tensors whose first axis is the worker; a worker's weights may lie anywhere at a constant stride (a
view of the rows of a packed ReplicaArena: `ReplicaArena.worker_tensor`).  The last axis is contiguous.  `stream` is a
raw cudaStream_t; None is torch's current stream of the tensors' device.  Outputs and workspaces that the caller does
not give are allocated for that stream.  Calls are asynchronous.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import struct
import threading
from typing import Dict, NamedTuple, Optional, Tuple, Union

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


# ---------------------------------------------------------------------------------------------- argument marshalling

_FFN_SHAPE = struct.Struct("=IiiiQQQ")                   # palsgd_ffn_shape
_QK_SHAPE = struct.Struct("=IiQIIIIiIQqd")               # palsgd_qk_shape
_WORDS = [struct.Struct(f"={n}q") for n in range(64)]


class _Args(threading.local):
    """The structs of one call, packed into one block of memory a thread: the shape at 0, matrices or heads from 64 on,
    the workspace size at the end.  The library reads them before it returns."""

    def __init__(self):
        self.mem = bytearray(640)
        self.keep = (C.c_char * len(self.mem)).from_buffer(self.mem)
        self.base = C.addressof(self.keep)
        self.size = C.c_size_t.from_buffer(self.mem, 632)


_args = _Args()


def _mats(*rows):
    """Packs operands (pointer and strides) behind the shape; their addresses, None for None."""
    m, at, words = _args, [], []
    base = m.base + 64
    for r in rows:
        if r is None:
            at.append(None)
        else:
            at.append(base + 8 * len(words))
            words += r
    _WORDS[len(words)].pack_into(m.mem, 64, *words)
    return at


def _refuse(where: str, why: str):
    raise PalsgdError(EINVAL, where, why)


def _check(rc: int, where: str) -> None:
    if rc:
        raise PalsgdError(rc, where, lib().palsgd_last_cuda_error(None).decode() if rc == -3 else "")


def _precision(t: torch.Tensor, where: str, name: str) -> int:
    dt = t.dtype
    if dt is torch.bfloat16:
        return PREC_BF16_MASTER
    if dt is torch.float32:
        return PREC_FP32
    _refuse(where, f"{name} must be float32 or bfloat16, not {dt}")


def _tensor(t, where: str, name: str, shape, dtype, device) -> torch.Tensor:
    if (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.device == device
            and (t.stride()[-1] == 1 or shape[-1] <= 1 or t.numel() == 0)):
        return t
    if not isinstance(t, torch.Tensor):
        _refuse(where, f"{name} must be a tensor")
    if t.shape != shape:
        _refuse(where, f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype:
        _refuse(where, f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        _refuse(where, f"{name} must be on {device}, not {t.device}")
    _refuse(where, f"the last axis of {name} must be contiguous")


def _mat(t, where: str, name: str, shape, dtype, device):
    """The checked matrix (K, rows, cols) as (pointer, worker stride, row stride)."""
    _tensor(t, where, name, shape, dtype, device)
    s = t.stride()
    return t.data_ptr(), s[0], s[1]


def _cuda(t, where: str, name: str, ndim: int) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(where, f"{name} must be a CUDA tensor")
    if t.dim() != ndim:
        _refuse(where, f"{name} must have {ndim} axes, not {t.dim()}")
    return t.device


class _On:
    """The device and the stream of a call: `raw` is the cudaStream_t; allocations inside the block belong to it."""
    __slots__ = ("device", "stream", "stack", "raw")

    def __init__(self, device: torch.device, stream: Optional[int]):
        self.device, self.stream, self.stack = device, stream, None

    def __enter__(self) -> "_On":
        index = self.device.index
        current = torch._C._cuda_getCurrentRawStream(index)
        other = self.stream is not None and self.stream != current
        self.raw = self.stream if other else current
        if other or torch._C._cuda_getDevice() != index:
            self.stack = contextlib.ExitStack()
            self.stack.enter_context(torch.cuda.device(self.device))
            if other:
                # stream 0 is the legacy default stream, which torch knows as its default stream
                self.stack.enter_context(torch.cuda.stream(
                    torch.cuda.ExternalStream(self.stream, self.device) if self.stream
                    else torch.cuda.default_stream(self.device)))
        return self

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()


_need: Dict[tuple, int] = {}              # workspace bytes by entry point and sizes, as last reported by the library


def _workspace(call, key: tuple, given: Optional[torch.Tensor], like: torch.Tensor, where: str):
    """call(workspace address, address of its size).  Without a workspace of the caller's, one of the size that such a
    call last asked for is allocated; the library reports the size that it wants where that is too small (operands that
    are not aligned need more)."""
    size, at = _args.size, _args.base + 632
    if given is not None:
        if given.dtype != torch.uint8 or given.device != like.device or not given.is_contiguous():
            _refuse(where, f"workspace must be a contiguous uint8 tensor on {like.device}")
        size.value = given.numel()
        _check(call(given.data_ptr(), at), where)
        return
    have = _need.get(key)
    if have is None:
        size.value = 0
        _check(call(None, at), where)
        have = size.value
    while True:
        ws = torch.empty(max(have, 1), dtype=torch.uint8, device=like.device)
        size.value = have
        rc = call(ws.data_ptr(), at)
        if rc != EINVAL or size.value <= have:
            break
        have = size.value
    _check(rc, where)
    if len(_need) > 4096:
        _need.clear()
    _need[key] = have


def block_status(stream: Optional[int] = None) -> None:
    """palsgd_block_status: raises PalsgdError if a matrix kernel's bounded wait gave up since the last call (its outputs
    are then unspecified).  Synchronises the stream."""
    raw = torch.cuda.current_stream().cuda_stream if stream is None else stream
    _check(lib().palsgd_block_status(C.c_void_p(raw)), "palsgd_block_status")


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints

def _groups(cols: int) -> int:
    return (cols + ACT8_GROUP - 1) // ACT8_GROUP


def _rows(t: torch.Tensor):
    """(rows, cols) or (K, rows, cols) as (pointer, worker stride, row stride)."""
    s = t.stride()
    return (t.data_ptr(), s[0], s[1]) if len(s) == 3 else (t.data_ptr(), 0, s[0])


def _act8(where, a: Act8, name, shape, dev):
    """The checked checkpoint of a (K, rows, cols) matrix as two triples."""
    return (_mat(a.q, where, name + ".q", shape, torch.int8, dev),
            _mat(a.exponent, where, name + ".exponent", (*shape[:-1], _groups(shape[-1])), torch.uint8, dev))


def _act8_run(entry: str, prec: int, x: torch.Tensor, a: Act8, raw: int, order) -> None:
    shape = x.shape
    at = _mats(_rows(x), _rows(a.q), _rows(a.exponent))
    k, r = (1, shape[0]) if len(shape) == 2 else (shape[0], shape[1])
    _check(getattr(lib(), entry)(prec, k, r, shape[-1], at[order[0]], at[order[1]], at[order[2]], raw), entry)


def act8_pack(x: torch.Tensor, *, out: Optional[Act8] = None, stream: Optional[int] = None) -> Act8:
    """palsgd_act8_pack: the 8-bit checkpoint of x (rows, cols) or (K, rows, cols), float32 or bfloat16."""
    where = "palsgd_act8_pack"
    dev = _cuda(x, where, "x", 2 if isinstance(x, torch.Tensor) and x.dim() == 2 else 3)
    prec, shape = _precision(x, where, "x"), x.shape
    _tensor(x, where, "x", shape, x.dtype, dev)
    groups = (*shape[:-1], _groups(shape[-1]))
    with _On(dev, stream) as on:
        if out is None:
            out = Act8(x.new_empty(shape, dtype=torch.int8), x.new_empty(groups, dtype=torch.uint8), x.dtype)
        else:
            _tensor(out.q, where, "out.q", shape, torch.int8, dev)
            _tensor(out.exponent, where, "out.exponent", groups, torch.uint8, dev)
        _act8_run(where, prec, x, out, on.raw, (0, 1, 2))
    return out


def act8_unpack(a: Act8, *, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                stream: Optional[int] = None) -> torch.Tensor:
    """palsgd_act8_unpack: the values that a checkpoint stands for, in `dtype` (default: the type it was taken from).
    They have at most eight significant bits: bfloat16 holds them exactly."""
    where = "palsgd_act8_unpack"
    q = a.q
    dev = _cuda(q, where, "q", 2 if isinstance(q, torch.Tensor) and q.dim() == 2 else 3)
    shape = q.shape
    _tensor(q, where, "q", shape, torch.int8, dev)
    _tensor(a.exponent, where, "exponent", (*shape[:-1], _groups(shape[-1])), torch.uint8, dev)
    with _On(dev, stream) as on:
        if out is None:
            out = q.new_empty(shape, dtype=dtype or a.dtype)
        else:
            _tensor(out, where, "out", shape, dtype or out.dtype, dev)
        _act8_run(where, _precision(out, where, "out"), out, a, on.raw, (1, 2, 0))
    return out


# ---------------------------------------------------------------------------------------------- gated feed-forward

def _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev):
    F = w_gate.shape[1] if isinstance(w_gate, torch.Tensor) and w_gate.dim() == 3 else 0
    return (F, _mat(w_gate, where, "w_gate", (K, F, D), dt, dev), _mat(w_up, where, "w_up", (K, F, D), dt, dev),
            _mat(w_down, where, "w_down", (K, D, F), dt, dev))


def _saved(where, save, saved, shape, dt, dev):
    """gate, up and their exponents as triples, or None."""
    if save == SAVE_NONE:
        return None, None, None, None
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    gate, up = saved
    if save == SAVE_8BIT:
        if not (isinstance(gate, Act8) and isinstance(up, Act8)):
            _refuse(where, "gate and up must both be Act8")
        (gq, ge), (uq, ue) = _act8(where, gate, "gate", shape, dev), _act8(where, up, "up", shape, dev)
        return gq, uq, ge, ue
    return _mat(gate, where, "gate", shape, dt, dev), _mat(up, where, "up", shape, dt, dev), None, None


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
    K, M, D = xs = x.shape
    mx = _mat(x, where, "x", xs, dt, dev)
    F, mg, mu, md = _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev)
    with _On(dev, stream) as on:
        y = x.new_empty(xs) if out is None else out
        my = _mat(y, where, "out", xs, dt, dev)
        if save == SAVE_NONE:
            saved = None
        elif saved is None:
            if save == SAVE_8BIT:
                G = _groups(F)
                saved = tuple([Act8(x.new_empty((K, M, F), dtype=torch.int8), x.new_empty((K, M, G), dtype=torch.uint8), dt)
                               for _ in range(2)])
            else:
                saved = (x.new_empty((K, M, F)), x.new_empty((K, M, F)))
        at = _mats(mx, mg, mu, md, my, *_saved(where, save, saved, (K, M, F), dt, dev))
        _FFN_SHAPE.pack_into(_args.mem, 0, K, prec, activation, save, M, D, F)
        entry, s = lib().palsgd_ffn_forward, _args.base
        _workspace(lambda ws, n: entry(s, *at, ws, n, on.raw), (where, K, M, D, F, prec), workspace, x, where)
    return y, saved


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
    K, M, D = ys = dy.shape
    mdy = _mat(dy, where, "dy", ys, dt, dev)
    F, mg, mu, md = _ffn_weights(where, w_gate, w_up, w_down, K, D, dt, dev)
    if not isinstance(saved, (tuple, list)) or len(saved) != 2:
        _refuse(where, "saved must be the pair (gate, up)")
    save = SAVE_8BIT if isinstance(saved[0], Act8) else SAVE_FULL
    if isinstance(x, Act8):
        if save != SAVE_8BIT:
            _refuse(where, "x may be an Act8 only where gate and up are")
        mx, me = _act8(where, x, "x", ys, dev)
    else:
        mx, me = _mat(x, where, "x", ys, dt, dev), None
    with _On(dev, stream) as on:
        want = (ys, (K, F, D), (K, F, D), (K, D, F))
        outs = list(out) if out is not None else [None] * 4
        if len(outs) != 4:
            _refuse(where, "out must be (dx, dw_gate, dw_up, dw_down)")
        mats = [None] * 4
        for i, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
            if i == 0 and not need_dx:
                outs[0] = None
                continue
            if outs[i] is None:
                outs[i] = dy.new_empty(want[i])
            mats[i] = _mat(outs[i], where, name, want[i], dt, dev)
        at = _mats(mdy, mx, me, mg, mu, md, *_saved(where, save, saved, (K, M, F), dt, dev), *mats)
        _FFN_SHAPE.pack_into(_args.mem, 0, K, prec, activation, save, M, D, F)
        entry, s = lib().palsgd_ffn_backward, _args.base
        _workspace(lambda ws, n: entry(s, *at, ws, n, on.raw), (where, K, M, D, F, prec, need_dx, me is None), workspace,
                   dy, where)
    return tuple(outs)


# ---------------------------------------------------------------------------------------------- q/k norm + rotation

def _heads(t, where: str, name: str, shape, dtype, device):
    """The checked heads (K, tokens, heads, head_dim) as (pointer, worker, token and head stride)."""
    _tensor(t, where, name, shape, dtype, device)
    s = t.stride()
    return t.data_ptr(), s[0], s[1], s[2]


def _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved):
    """Checks the arguments and packs the shape; the packed operands, and the addresses of the tables."""
    dev = _cuda(q, where, "q", 4)
    prec, dt = _precision(q, where, "q"), q.dtype
    K, M, HQ, DH = q.shape
    HK = k.shape[2] if isinstance(k, torch.Tensor) and k.dim() == 4 else -1
    ops = [_heads(q, where, "q", q.shape, dt, dev), _heads(k, where, "k", (K, M, HK, DH), dt, dev)]
    for name, w in (("w_q", w_q), ("w_k", w_k)):
        _tensor(w, where, name, (K, DH), dt, dev)
        ops.append((w.data_ptr(), w.stride(0), 0))
    if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
        _refuse(where, "cos must be a (rows, rotary_dim / 2) tensor")
    rows, half = shape = cos.shape
    for name, t in (("cos", cos), ("sin", sin)):
        if not _tensor(t, where, name, shape, torch.float32, dev).is_contiguous():
            _refuse(where, f"{name} must be contiguous")
    _tensor(positions, where, "positions", (K, M), torch.int32, dev)
    _QK_SHAPE.pack_into(_args.mem, 0, K, prec, M, HQ, HK, DH, 2 * half, 1 if interleaved else 0, 0, rows,
                        positions.stride(0) if K > 1 else 0, eps)
    return dev, ops, (cos.data_ptr(), sin.data_ptr(), positions.data_ptr())


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[int] = None):
    """palsgd_qk_norm_rope_forward: RMS norm of every head of q (K, tokens, heads_q, head_dim) and k, with weights
    w_q, w_k (K, head_dim), then the rotation of the first 2*cos.shape[1] values by the angle tables cos, sin
    (rows, rotary_dim / 2) at positions (K, tokens) int32.  Returns (q_out, k_out)."""
    where = "palsgd_qk_norm_rope_forward"
    dev, ops, tables = _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    with _On(dev, stream) as on:
        out = (q.new_empty(q.shape), k.new_empty(k.shape)) if out is None else tuple(out)
        mq, mk, mwq, mwk, mo, mp = _mats(*ops, _heads(out[0], where, "q_out", q.shape, q.dtype, dev),
                                         _heads(out[1], where, "k_out", k.shape, q.dtype, dev))
        _check(lib().palsgd_qk_norm_rope_forward(_args.base, mq, mk, mwq, mwk, *tables, mo, mp, on.raw), where)
    return out


def qk_norm_rope_backward(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
                          positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False,
                          out: Optional[Tuple] = None, workspace: Optional[torch.Tensor] = None,
                          stream: Optional[int] = None):
    """palsgd_qk_norm_rope_backward: (dq, dk, dw_q, dw_k) from the gradients of qk_norm_rope's results and its inputs.
    `out` gives the memory to write to; entries may be None."""
    where = "palsgd_qk_norm_rope_backward"
    dev, ops, tables = _qk(where, q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    dt = q.dtype
    grads = [_heads(dq_out, where, "dq_out", q.shape, dt, dev), _heads(dk_out, where, "dk_out", k.shape, dt, dev)]
    with _On(dev, stream) as on:
        outs = list(out) if out is not None else [None] * 4
        if len(outs) != 4:
            _refuse(where, "out must be (dq, dk, dw_q, dw_k)")
        mats = []
        for i, (name, like) in enumerate((("dq", q), ("dk", k), ("dw_q", w_q), ("dw_k", w_k))):
            if outs[i] is None:
                outs[i] = like.new_empty(like.shape)
            if i < 2:
                mats.append(_heads(outs[i], where, name, like.shape, dt, dev))
            else:
                _tensor(outs[i], where, name, like.shape, dt, dev)
                mats.append((outs[i].data_ptr(), outs[i].stride(0), 0))
        at = _mats(*grads, *ops, *mats)
        entry, s = lib().palsgd_qk_norm_rope_backward, _args.base
        _workspace(lambda ws, n: entry(s, *at[:6], *tables, *at[6:], ws, n, on.raw), (where, *q.shape, k.shape[2]),
                   workspace, q, where)
    return tuple(outs)
