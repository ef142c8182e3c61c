"""MI355X (gfx950) differentiable finite-difference PDE residual operator.

Three C-ABI entry points (include/fpde.h), implemented as hand-written HIP
kernels in ``csrc/`` and exposed here through a thin ctypes binding:
``fpde_residual_fwd`` (fused stencil + mean-squared loss),
``fpde_residual_bwd`` (interior analytic adjoint, gather form) and
``fpde_bc_correct`` (boundary-gradient correction).  ``workloads`` holds the
seeded synthetic inputs of the five benchmark operators.

``network`` holds the operators of the networks whose fields the residuals
judge (include/fpde_net.h): norm, causal convolution and selective scan along
time, orthogonalised weight updates.
"""
from . import workloads  # noqa: F401

__all__ = ["workloads", "binding", "network"]


def __getattr__(name):
    # the bindings load the built libraries; import them lazily so that the workload
    # generators stay usable on machines without them
    if name in ("binding", "network"):
        import importlib  # noqa: PLC0415
        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
