"""B200-native evolution-strategy generation (ask -> rollout -> tell) behind a C-ABI.

``operators`` holds the calls that need no solver; ``binding`` is the thin ctypes layer over ``libevo.so``; ``workloads`` holds the synthetic
configurations and seeded input generators; ``build`` compiles the CUDA sources.
"""
from .binding import EvoConfig, EvoError, Solver, load_library  # noqa: F401
from .operators import (combine_rows, combine_rows_backward, grouped_linear, grouped_linear_backward, mlp_actions, muon_step,  # noqa: F401
                        orthogonalize, policy_loss, route_rows, take_rows)
from . import workloads  # noqa: F401
