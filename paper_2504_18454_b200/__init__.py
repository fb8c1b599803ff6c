"""PALSGD update / synchronisation path for NVIDIA B200 (sm_100a).

`Palsgd` is a thin ctypes binding over the C ABI in `include/palsgd.h`
(`libpalsgd.so`, built in-tree by `paper_2504_18454_b200.build`).  Every step of
the path runs in the library's CUDA kernels; this package only marshals
arguments.  PyTorch supplies device memory and streams.  `block` binds the
operators with which the K workers make their gradients (`include/palsgd_block.h`).
"""
from .binding import (  # noqa: F401
    Palsgd,
    PalsgdError,
    decision,
    plan_layout,
    schedule_value,
    OUTER_SGD,
    OUTER_ADAMW,
    SCHED_WARMUP_CONSTANT,
    SCHED_WARMUP_COSINE,
    outer_sync_noalloc,
    NOALLOC_SCRATCH_BYTES,
    lib,
    strerror,
    INNER_ADAMW,
    INNER_SGDM,
    PREC_FP32,
    PREC_BF16_MASTER,
    TUNE_INNER_GRID_CAP,
    TUNE_OUTER_GRID_CAP,
    TUNE_INNER_VARIANT,
    TUNE_OUTER_SUB_ELEMS,
    TUNE_DDP_SUB_ELEMS,
    TUNE_DDP_VARIANT,
    TUNE_OUTER_VARIANT,
    TUNE_OUTER_DYNAMIC,
)

# The block operators take torch tensors: `block`, and torch with it, is imported where one of its names is first used.
_BLOCK = (
    "Act8", "act8_pack", "act8_unpack", "block_status", "ffn_backward", "ffn_forward", "qk_norm_rope",
    "qk_norm_rope_backward", "linear_forward", "linear_backward", "layer_norm_forward", "layer_norm_backward",
    "cross_entropy_forward", "cross_entropy_backward", "ACT_NONE", "ACT8_GROUP", "ACT_GELU", "ACT_GELU_TANH", "ACT_RELU", "ACT_SILU", "SAVE_8BIT", "SAVE_FULL",
    "SAVE_NONE",
)
__all__ = [n for n in globals() if not n.startswith("_")] + ["block", *_BLOCK]


def __getattr__(name):
    if name != "block" and name not in _BLOCK:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from importlib import import_module
    block = import_module(".block", __name__)
    globals().update((n, getattr(block, n)) for n in _BLOCK)
    return globals()[name]                               # (importing a submodule sets `block` itself)


def __dir__():
    return sorted({*globals(), *__all__})
