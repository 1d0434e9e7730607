"""Streaming-rollout frame update on B200: Python binding of the C-ABI CUDA library.

The package holds the CUDA sources (csrc/), their build step (build.py) and a thin
ctypes binding (binding.py) with the same names as the C entry points.  Every step
of the frame update runs in the library's kernels; Python only marshals arguments.
operators.py binds the operators of the temporal head that may stand behind a rollout.
"""
from .binding import Graph, SrError, load_library, STATUS  # noqa: F401


_OPERATORS = ("Microscaled", "TemporalHead", "linear_attention_run", "linear_attention_step", "operator_reset", "operator_status", "product", "quantize", "rms_norm")


def __getattr__(name):
    # the operators' module needs torch, which a theory-only graph does not
    if name in _OPERATORS:
        from . import operators
        value = getattr(operators, name)
        globals()[name] = value
        return value
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
