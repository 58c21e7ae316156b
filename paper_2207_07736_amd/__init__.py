"""GPU-vectorised, kernel-fused RL data collection for MI355X (gfx950).

The compute path is librlsim.so (hand-written HIP kernels behind the C ABI of
include/rlsim.h); ``rlsim`` is its thin ctypes binding and ``head`` that of the
output head's operators.  Importing this package loads the library and fails if it
has not been built.
"""
from .rlsim import *  # noqa: F401,F403
from .rlsim import EXPORTS, LIB_PATH, RlsimError, Simulator, Trajectory, TrajRows, stats_only  # noqa: F401
from .head import (Head, rlsim_distill, rlsim_head_create, rlsim_head_destroy, rlsim_head_distill,  # noqa: F401
                   rlsim_head_last_error, rlsim_head_sample, rlsim_sample)
