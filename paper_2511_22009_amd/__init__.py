"""Stream-batched rectified-flow step on MI355X (gfx950): Python binding of
libstreamflow.so. Every computation runs in the library's HIP kernels; this package
marshals arguments (torch tensors provide device memory and streams)."""
from importlib.util import find_spec

from .binding import (Buffer, Cond, KernelClass, Model, SFError, Precision, lib_path, load_library,
                      library_symbols)

# the operators on torch tensors; importing the package itself needs no torch
_OPERATORS = ("Rotary", "gated_matmul_f8", "matmul_f8", "matmul_i8", "qk_norm_rotate", "quantize_f8", "quantize_rows",
              "residual_norm", "rotate")

__all__ = ["Buffer", "Cond", "KernelClass", "Model", "SFError", "Precision", "lib_path", "load_library",
           "library_symbols"]
if all(find_spec(n) for n in ("torch", __name__ + "._operators")):
    __all__ += _OPERATORS  # `import *` loads them, so they are named only where that works


def __getattr__(name):
    if name in _OPERATORS:
        from . import operators
        globals().update({n: getattr(operators, n) for n in _OPERATORS})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
