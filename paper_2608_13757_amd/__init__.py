"""Barrier-free synchronization of loop-nested multi-engine kernels on MI355X.

The product is the C-ABI library ``libbfs.so`` (header ``include/bfs.h``):
a host planner for the thresholds of the paper's per-loop allocation and HIP
kernels for gfx950 whose engines are specialised wavefronts synchronising
through LDS counters.  ``bfs`` is the thin ctypes binding; ``ops`` binds the operators
beside the plans (a mixture of experts' router, dispatch and combination, the
global gradient norm)."""
from .bfs import (ALLOC_PER_ENGINE, ALLOC_PER_INSTR, ALLOC_PER_LOOP, KASE_FALLBACK, MODE_BARRIER, MODE_BARRIER_FREE,  # noqa: F401
                  BfsError, Plan, lib, parse_debug_log)

_OPS = ("GradSet", "grad_clip", "grad_norm", "moe_combine", "moe_combine_grad", "moe_dispatch", "moe_dispatch_grad",
        "moe_dispatch_workspace", "moe_route", "moe_route_grad")


def __getattr__(name):
    """The operators, loaded at their first use (they import torch)."""
    if name in _OPS:
        from . import ops
        globals().update({n: getattr(ops, n) for n in _OPS})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
