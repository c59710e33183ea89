"""MI355X-native line-granularity network simulator (HIP kernels behind a C ABI).

``paper_2606_10440_amd.sim`` is the ctypes binding of ``libsimgpu.so``;
``paper_2606_10440_amd.ops``, its operators for an expert-parallel step on
torch tensors, is imported when it is first asked for, so that the simulator
needs no torch; ``paper_2606_10440_amd.build`` builds both.
"""
import importlib

from . import sim  # noqa: F401
from .sim import Simulator, SimError  # noqa: F401


def __getattr__(name):
    if name == "ops":
        return importlib.import_module(".ops", __name__)
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
