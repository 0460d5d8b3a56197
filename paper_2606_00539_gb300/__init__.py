"""GB300-native GNMR per-step monitor (sm_103a).

The monitor reduces every unit's gradient to its L2 norm, updates the unit's
historical mean and GNMR window, forms GNMR and Delta-GNMR, and selects at
most maxO units for the recovery path under the lock interval -- one CUDA
kernel launch per training step, behind the C ABI in ``include/gnmr.h``.

* :mod:`._native` -- ctypes binding with the C entry points' names.
* :class:`Monitor` -- torch-facing wrapper (torch supplies memory and streams).
* :class:`ExpertProducts`, :func:`expert_linear` -- the products of the units that the
  mask chooses a path for: 16-bit and 8-bit, grouped by expert, with their gradients.
* :mod:`.build` -- compiles ``libgnmr.so`` for sm_103a.
"""
from ._native import GnmrError, load  # noqa: F401
from .monitor import Monitor  # noqa: F401
from .products import ExpertProducts, expert_linear  # noqa: F401

__all__ = ["Monitor", "ExpertProducts", "expert_linear", "GnmrError", "load"]
