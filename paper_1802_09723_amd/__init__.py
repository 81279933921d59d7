"""MI355X-native Recurrent Residual Module: thin Python binding over the C-ABI HIP library.

The binding only marshals arguments (device pointers, shapes, the current HIP stream); every
step of the per-layer delta update runs in the library's gfx950 kernels.  There is no CPU or
PyTorch fallback: if the built library is missing, importing :mod:`.binding` symbols that need
it raises.
"""
from .binding import (  # noqa: F401
    BF16, BIN, CONV, FC, I8, Layer, RRMError, Shape, StackEntry, Stats, lib, lib_path, probe_copy, probe_mfma, relu_requant_pool_i8, stack_step,
)

# (operators imports torch, which takes a second or more: not before one of its names is asked for)
_OPERATORS = ("gated_ff", "gated_ff_backward", "gated_scan", "gated_scan_backward", "gated_scan_marks", "group_norm_act",
              "group_norm_act_backward", "group_norm_act_of")


def __getattr__(name):
    if name in _OPERATORS or name == "operators":
        from importlib import import_module
        module = import_module(".operators", __name__)
        globals().update({n: getattr(module, n) for n in _OPERATORS})
        return module if name == "operators" else getattr(module, name)
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted({*globals(), *_OPERATORS, "operators"})
